// The linear operator for few rows (decoding steps): what bounds it is reading w once, so w streams through
// the CUDA cores in whole 128-byte lines and no tensor-core tile is padded with empty rows.
//
// A block owns LC x 16 bytes of columns and a run of the contraction; its 256 threads are LC column groups by 256 / LC
// rows of w, each thread with N x (8 or 4) fp32 sums.  The runs of a column block form a cluster, whose blocks add
// their sums through distributed shared memory in a fixed order, so that the whole operator is one launch and the
// result has the same bits from run to run.  A second wave of blocks would double the time (each has some 3 us of
// its own: launch, staging of x, the joins), so the launcher aims just below two blocks per multiprocessor, with
// narrow column blocks (LC = 4) before runs that need a cluster.
// Measured (back to back, w from HBM): 1024 -> 8192 bf16 6.2 us for one row, 10 us for eight; 8192 -> 1024 7.6 us.  From
// three rows on (linear.cu) the tensor cores are as fast where one launch of theirs covers the product.
#include <algorithm>

#include "activation.cuh"
#include "checks.cuh"
#include "linear.cuh"
#include "pack.cuh"
#include "sm100_ptx.cuh"

namespace gshard {

namespace {

constexpr int kFewThreads = 256;
constexpr int kFewChunk = 512;          // rows of w per staging of x

struct FewArgs {
  const void* x; const void* w; void* y;
  LinearEpilogue lin;
  int* status;
  int n, K, cols, run;                  // run: contraction length per block of the cluster
};

__device__ __forceinline__ float4 ld_cluster(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
  return v;
}

// GATED: w holds the gate's columns and then the other factor's; the first half of a block's columns are gate columns, the second half
// the same columns of the other factor, and lin.act(gate) times that is the result.
template <typename T, typename TY, int N, int LC, bool GATED>
__global__ void __launch_bounds__(kFewThreads, 2) linear_few_kernel(const FewArgs a) {
  constexpr int W = 16 / (int)sizeof(T);            // columns per thread
  constexpr int CT = LC * W;                        // columns per block
  constexpr int RW = 32 / LC, RB = 8 * RW;          // rows of w per warp and per block
  constexpr int U = N == 8 ? 4 : 8;                 // rows of w per batch; the next batch is on its way meanwhile
  __shared__ __align__(16) float xs[N][kFewChunk];
  __shared__ __align__(16) float warp_sums[8][N][CT];
  __shared__ __align__(16) float sums[N][CT];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int splits = gridDim.y, rank = blockIdx.y;  // the cluster spans grid.y
  const int half_cols = a.cols / 2;
  const int lc = lane % LC;
  const int col = !GATED ? blockIdx.x * CT + lc * W : (lc < LC / 2 ? 0 : half_cols) + blockIdx.x * (CT / 2) + lc % (LC / 2) * W;
  const int k_row = warp * RW + lane / LC;
  const int k0 = rank * a.run, k1 = min(a.K, k0 + a.run);
  if (blockIdx.x == 0 && blockIdx.y == 0 && tid == 0) *a.status = 0;
  const T* x = static_cast<const T*>(a.x);
  const T* w = static_cast<const T*>(a.w);
  float acc[N][W];
#pragma unroll
  for (int r = 0; r < N; ++r)
#pragma unroll
    for (int j = 0; j < W; ++j) acc[r][j] = 0.f;
  const bool in = !GATED ? col < a.cols : blockIdx.x * (CT / 2) + lc % (LC / 2) * W < half_cols;
  for (int kc = k0; kc < k1; kc += kFewChunk) {
    const int len = min(kFewChunk, k1 - kc);
    // the chunk's first rows of w are on their way before x is staged
    Pack<T, W> p[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (in && k_row + RB * u < len) p[u].load_once(w + (long long)(kc + k_row + RB * u) * a.cols + col);
    if (kc != k0) __syncthreads();                   // the previous chunk of x has been read
    for (int i = tid; i < N * (kFewChunk / 8); i += kFewThreads) {
      const int r = i / (kFewChunk / 8), c = i % (kFewChunk / 8) * 8;
      if (c < len) {                                 // K is a multiple of 8, and so is len
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = 0.f;
        if (r < a.n) {
#pragma unroll
          for (int h = 0; h < 8; h += W) load_pack<T, W>(x + (long long)r * a.K + kc + c + h, f + h);
        }
        *reinterpret_cast<float4*>(&xs[r][c]) = make_float4(f[0], f[1], f[2], f[3]);
        *reinterpret_cast<float4*>(&xs[r][c + 4]) = make_float4(f[4], f[5], f[6], f[7]);
      }
    }
    __syncthreads();
    for (int k = k_row; k < len; k += RB * U) {
      Pack<T, W> q[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        q[u] = p[u];
        if (in && k + RB * (U + u) < len) p[u].load_once(w + (long long)(kc + k + RB * (U + u)) * a.cols + col);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (in && k + RB * u < len) {
          float f[W];
#pragma unroll
          for (int j = 0; j < W; ++j) f[j] = q[u].get(j);
#pragma unroll
          for (int r = 0; r < N; ++r) {
            const float xv = xs[r][k + RB * u];
#pragma unroll
            for (int j = 0; j < W; ++j) acc[r][j] = fmaf(xv, f[j], acc[r][j]);
          }
        }
      }
    }
  }
  // a warp's rows of w, then the warps, then the blocks of the cluster
#pragma unroll
  for (int r = 0; r < N; ++r)
#pragma unroll
    for (int j = 0; j < W; ++j) {
#pragma unroll
      for (int off = LC; off < 32; off <<= 1) acc[r][j] += __shfl_xor_sync(0xffffffffu, acc[r][j], off);
    }
  if (lane < LC) {
#pragma unroll
    for (int r = 0; r < N; ++r)
#pragma unroll
      for (int j = 0; j < W; j += 4)
        *reinterpret_cast<float4*>(&warp_sums[warp][r][lane * W + j]) = make_float4(acc[r][j], acc[r][j + 1], acc[r][j + 2], acc[r][j + 3]);
  }
  __syncthreads();
  for (int i = tid; i < N * CT; i += kFewThreads) {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) s += (&warp_sums[k][0][0])[i];
    (&sums[0][0])[i] = s;
  }
  if (splits > 1) ptx::cluster_sync_all();
  else __syncthreads();
  // every block of the cluster finishes its share of the outputs, four columns at a time
  auto total = [&](int r, int c) {
    if (splits == 1) return *reinterpret_cast<const float4*>(&sums[r][c]);
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    const uint32_t at = ptx::smem_u32(&sums[r][c]);
    for (int k = 0; k < splits; ++k) {
      const float4 v = ld_cluster(ptx::map_to_cta(at, k));
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    return s;
  };
  constexpr int CO = GATED ? CT / 2 : CT;
  const int out_cols = GATED ? half_cols : a.cols;
  for (int i = rank * kFewThreads + tid; i < N * CO / 4; i += splits * kFewThreads) {
    const int r = i / (CO / 4), c = i % (CO / 4) * 4;
    const int out_col = blockIdx.x * CO + c;
    if (r >= a.n || out_col >= out_cols) continue;
    const float4 s = total(r, c);
    if constexpr (GATED) gated_epilogue4<TY>(a.lin, a.y, r, half_cols, out_col, s, total(r, CO + c));
    else linear_epilogue4<TY>(a.lin, a.y, (long long)r * a.cols + out_col, out_col, s);
  }
  if (splits > 1) ptx::cluster_sync_all();           // no block leaves while another may still read its sums
}

template <typename T, typename TY, int N, int LC, bool GATED>
int launch_few_t(const FewArgs& a, int blocks, int splits, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(blocks, splits, 1);
  cfg.blockDim = dim3(kFewThreads, 1, 1);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 1;
  attr[0].val.clusterDim.y = splits;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = splits > 1 ? 1 : 0;
  if (cudaLaunchKernelEx(&cfg, linear_few_kernel<T, TY, N, LC, GATED>, a) != cudaSuccess) { cudaGetLastError(); return GSHARD_ERR_CUDA; }
  count_launch();
  return GSHARD_OK;
}

template <typename T, typename TY, int N, bool GATED>
int launch_few_n(const FewArgs& a, int lc, int splits, cudaStream_t st) {
  const int blocks = ceil_div(a.cols, lc * 16 / (int)sizeof(T));
  return lc == 8 ? launch_few_t<T, TY, N, 8, GATED>(a, blocks, splits, st) : launch_few_t<T, TY, N, 4, GATED>(a, blocks, splits, st);
}

template <typename T, typename TY, bool GATED>
int launch_few(const FewArgs& a, int lc, int splits, cudaStream_t st) {
  if (a.n == 1) return launch_few_n<T, TY, 1, GATED>(a, lc, splits, st);
  if (a.n == 2) return launch_few_n<T, TY, 2, GATED>(a, lc, splits, st);
  if (a.n <= 4) return launch_few_n<T, TY, 4, GATED>(a, lc, splits, st);
  return launch_few_n<T, TY, 8, GATED>(a, lc, splits, st);
}

}  // namespace

int launch_linear_few(int n, int K, int cols, bool bf16, bool out_f32, const void* x, const void* w, void* y,
                      const LinearEpilogue& lin, int* status, cudaStream_t st, bool gated) {
  const int wide = ceil_div(cols, bf16 ? 64 : 32), room = 2 * 148;
  const int lc = 2 * wide <= room ? 4 : 8;
  const int blocks = lc == 4 ? 2 * wide : wide;
  int splits = 1;
  while (splits < 8 && 2 * blocks * splits <= room && K / (2 * splits) >= 128) splits *= 2;
  FewArgs a{x, w, y, lin, status, n, K, cols, ceil_div(ceil_div(K, splits), 32) * 32};
  if (gated) return bf16 ? launch_few<__nv_bfloat16, __nv_bfloat16, true>(a, lc, splits, st) : launch_few<float, float, true>(a, lc, splits, st);
  if (bf16) return out_f32 ? launch_few<__nv_bfloat16, float, false>(a, lc, splits, st)
                           : launch_few<__nv_bfloat16, __nv_bfloat16, false>(a, lc, splits, st);
  return launch_few<float, float, false>(a, lc, splits, st);
}

}  // namespace gshard
