// Cross attention of a decoding step: a few rows (queries times the heads that share a key head) against a long source.  What bounds it
// is reading k and v once, so both stream through the CUDA cores straight into registers, and no tile of 128 rows is padded.
//
// A group of LPR lanes owns a key: a lane holds 16 bytes of it, and of the value beside it, and the same part of every row's
// query and output.  A batch of U keys per group is in flight: partial products over the lane's 16 bytes, added over the group by
// shuffles, then one step of the running maximum and sum for the whole batch.  Groups, warps and - where the batch alone does not
// fill the GPU - up to 8 blocks of a cluster take keys in turns; their (maximum, sum, output) are joined in a fixed order through
// shuffles, shared memory and distributed shared memory, so the operator is one launch and has the same bits from run to run.
// 96 sources of up to 1024 keys, 16 heads of 128, bf16: 86 to 96 us, 5.7 to 6.3 TB/s.
#include <algorithm>

#include "attention.cuh"
#include "pack.cuh"
#include "sm100_ptx.cuh"

namespace gshard {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxSplits = 8;

__device__ __forceinline__ float ld_cluster_f32(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr));
  return v;
}

template <int LPR>
__device__ __forceinline__ float over_group(float v) {
#pragma unroll
  for (int off = LPR / 2; off; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
  return v;
}

template <typename T, int LPR, int R>
__global__ void __launch_bounds__(kThreads, R == 1 ? 4 : R == 2 ? 3 : R == 4 ? 2 : 1) attention_few_kernel(const AttentionArgs a, int rows, int splits) {
  constexpr int W = 16 / (int)sizeof(T);           // elements per lane
  constexpr int DP = LPR * W, G = 32 / LPR;        // groups of a warp
  constexpr int U = R <= 2 ? 4 : 2;                // keys of a group per batch
  __shared__ float s_out[kWarps][R][DP];
  __shared__ float s_top[kWarps][R], s_sum[kWarps][R];
  __shared__ float c_out[R][DP], c_top[R], c_sum[R];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int part = lane % LPR, grp = lane / LPR;
  const int rank = blockIdx.x % splits, kh = blockIdx.x / splits % a.Hkv, b = blockIdx.x / splits / a.Hkv;
  const int len = source_length(a, b);
  const int share = ((len + splits - 1) / splits + 15) / 16 * 16;       // keys per block
  const int begin = min(len, rank * share), end = min(len, begin + share);
  const int d = part * W;
  const bool live = d < a.D;
  const float c = a.scale * kLog2e;
  float q[R][W], out[R][W], top[R], sum[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    top[r] = -INFINITY;
    sum[r] = 0.f;
#pragma unroll
    for (int j = 0; j < W; ++j) q[r][j] = out[r][j] = 0.f;
    if (r < rows && live) {
      const int h = kh * (a.H / a.Hkv) + r / a.Tq, t = r % a.Tq;
      load_pack<T, W>(static_cast<const T*>(a.q) + ((long long)b * a.Tq + t) * a.q_stride + (long long)h * a.D + d, q[r]);
    }
  }
  const T* k = static_cast<const T*>(a.k) + (long long)b * a.Tk * a.k_stride + (long long)kh * a.D + d;
  const T* v = static_cast<const T*>(a.v) + (long long)b * a.Tk * a.v_stride + (long long)kh * a.D + d;
  const int me = warp * G + grp;                   // of kWarps * G groups
  for (int base = begin; base < end; base += kWarps * G * U) {
    Pack<T, W> pk[U], pv[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int key = base + u * kWarps * G + me;
      pk[u].raw = pv[u].raw = make_uint4(0, 0, 0, 0);
      if (key < end && live) {
        pk[u].load_once(k + key * a.k_stride);
        pv[u].load_once(v + key * a.v_stride);
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float s[U], m = top[r];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float x = 0.f;
#pragma unroll
        for (int j = 0; j < W; ++j) x = fmaf(q[r][j], pk[u].get(j), x);
        x = over_group<LPR>(x);
        s[u] = base + u * kWarps * G + me < end ? x : -INFINITY;
        m = fmaxf(m, s[u]);
      }
      const float ref = m == -INFINITY ? 0.f : m;
      const float shrink = exp2f((top[r] - ref) * c);
      top[r] = m;
      float t = 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        s[u] = exp2f((s[u] - ref) * c);        // c here, not in q: that product may be beyond fp32
        t += s[u];
      }
      sum[r] = fmaf(sum[r], shrink, t);
#pragma unroll
      for (int j = 0; j < W; ++j) {
        float o = out[r][j] * shrink;
#pragma unroll
        for (int u = 0; u < U; ++u) o = fmaf(s[u], pv[u].get(j), o);
        out[r][j] = o;
      }
    }
  }
  // the groups of a warp, then the warps, then the blocks: each part is scaled to the common maximum
#pragma unroll
  for (int r = 0; r < R; ++r) {
#pragma unroll
    for (int off = LPR; off < 32; off <<= 1) {
      const float other = __shfl_xor_sync(0xffffffffu, top[r], off);
      const float m = fmaxf(top[r], other), ref = m == -INFINITY ? 0.f : m;
      const float mine = exp2f((top[r] - ref) * c);
      top[r] = m;
      // both sides add the same two terms, in the same order
      sum[r] *= mine;
      const float os = __shfl_xor_sync(0xffffffffu, sum[r], off);
      sum[r] = sum[r] + os;
#pragma unroll
      for (int j = 0; j < W; ++j) {
        out[r][j] *= mine;
        out[r][j] += __shfl_xor_sync(0xffffffffu, out[r][j], off);
      }
    }
    if (grp == 0) {
#pragma unroll
      for (int j = 0; j < W; ++j) s_out[warp][r][d + j] = out[r][j];
      if (part == 0) { s_top[warp][r] = top[r]; s_sum[warp][r] = sum[r]; }
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < R * DP; i += kThreads) {
    const int r = i / DP, col = i % DP;
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) m = fmaxf(m, s_top[w][r]);
    const float ref = m == -INFINITY ? 0.f : m;
    float o = 0.f, t = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float f = exp2f((s_top[w][r] - ref) * c);
      o = fmaf(s_out[w][r][col], f, o);
      t = fmaf(s_sum[w][r], f, t);
    }
    c_out[r][col] = o;
    if (col == 0) { c_top[r] = m; c_sum[r] = t; }
  }
  if (splits > 1) ptx::cluster_sync_all();
  else __syncthreads();
  // every block finishes its share of the outputs, two neighbouring columns per thread
  for (int i = rank * kThreads + threadIdx.x; i < R * DP / 2; i += splits * kThreads) {
    const int r = i / (DP / 2), col = i % (DP / 2) * 2;
    if (r >= rows || col >= a.D) continue;
    float o[2], t, m;
    if (splits == 1) {
      o[0] = c_out[r][col]; o[1] = c_out[r][col + 1]; t = c_sum[r]; m = c_top[r];
    } else {
      const uint32_t at_top = ptx::smem_u32(&c_top[r]), at_sum = ptx::smem_u32(&c_sum[r]), at_out = ptx::smem_u32(&c_out[r][col]);
      m = -INFINITY;
      for (int w = 0; w < splits; ++w) m = fmaxf(m, ld_cluster_f32(ptx::map_to_cta(at_top, w)));
      const float ref = m == -INFINITY ? 0.f : m;
      o[0] = o[1] = t = 0.f;
      for (int w = 0; w < splits; ++w) {
        const float f = exp2f((ld_cluster_f32(ptx::map_to_cta(at_top, w)) - ref) * c);
        o[0] = fmaf(ld_cluster_f32(ptx::map_to_cta(at_out, w)), f, o[0]);
        o[1] = fmaf(ld_cluster_f32(ptx::map_to_cta(at_out + 4, w)), f, o[1]);
        t = fmaf(ld_cluster_f32(ptx::map_to_cta(at_sum, w)), f, t);
      }
    }
    const float factor = len ? 1.f / t : 0.f;
    o[0] *= factor; o[1] *= factor;
    const int h = kh * (a.H / a.Hkv) + r / a.Tq, q_row = r % a.Tq;
    store_pack<T, 2>(static_cast<T*>(a.o) + (((long long)b * a.Tq + q_row) * a.H + h) * a.D + col, o);
    if (a.lse && col == 0) a.lse[((long long)b * a.H + h) * a.Tq + q_row] = len ? m * a.scale + logf(t) : -INFINITY;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = 0;
  if (splits > 1) ptx::cluster_sync_all();         // no block leaves while another may still read its parts
}

template <typename T, int LPR, int R>
int launch_few_t(const AttentionArgs& a, int rows, int splits, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(a.B * a.Hkv * splits, 1, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = splits;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = splits > 1 ? 1 : 0;
  if (cudaLaunchKernelEx(&cfg, attention_few_kernel<T, LPR, R>, a, rows, splits) != cudaSuccess) { cudaGetLastError(); return GSHARD_ERR_CUDA; }
  count_launch();
  return GSHARD_OK;
}

template <typename T, int LPR>
int launch_few(const AttentionArgs& a, int rows, int splits, cudaStream_t st) {
  if (rows == 1) return launch_few_t<T, LPR, 1>(a, rows, splits, st);
  if (rows == 2) return launch_few_t<T, LPR, 2>(a, rows, splits, st);
  if (rows <= 4) return launch_few_t<T, LPR, 4>(a, rows, splits, st);
  return launch_few_t<T, LPR, 8>(a, rows, splits, st);
}

}  // namespace

// Whether this kernel takes the call.  It never spreads a key head over more than a cluster, the other kernels cut the source into parts,
// but take tiles of 64 (fp32) or 128 rows.
// bf16: by what it measured beside the tensor cores' (which take any number of rows alike), us, key heads of 128 x keys:
//   rows                 1           2           4           8
//   16 x 512         5.8 / 14.9  6.7 / 15    9.3 / 15   20.8 / 15
//   128 x 512        9.4 / 16.5 15.6 / 17   21.8 / 17   51.7 / 17
//   1024 x 2048      157 / 203   173 / 205   329 / 205   702 / 205
//   16 x 32768        87 / 68    104 / 68    176 / 68    389 / 68
// fp32: by estimates in us, fitted to what both kernels measured at 1 to 64 key heads and 2048 to 65536 keys: here the time of a block's keys
// (5 to 8 rows run in two rounds from 9 key heads on); there a least, all tiles' time, and that of the join of the parts.  Over those 80
// sizes with 1, 2, 4 and 8 rows the choice took at most a tenth longer than the better of the two.
// Key heads of 128 x keys, as queries of one head per key head:
//   rows                 1           2           4           8
//   1 x 4096        12.6 / 47   15.6 / 47   24.6 / 47   35.5 / 47
//   1 x 32768        120 / 82    138 / 85    230 / 84    301 / 86
//   4 x 8192          34 / 56     39 / 57     64 / 58     85 / 58
//   4 x 32768        123 / 142   141 / 144   236 / 145   314 / 146
//   16 x 8192         38 / 141    46 / 142    75 / 141   166 / 142
//   64 x 16384       155 / 998   203 / 998   293 / 998   790 / 998
bool attention_is_few(bool bf16, int B, int Tq, int Tk, int H, int Hkv, int D) {
  const long long rows = (long long)Tq * (H / Hkv), heads = (long long)B * Hkv;
  if (rows > 8) return false;
  if (bf16) {
    if (rows <= 2) return Tk <= 16384 || heads >= 64;
    return heads <= 32 && Tk * rows <= (rows <= 4 ? 8192 : 2048);
  }
  if (heads > 16) return true;
  const double width = D <= 64 ? 0.5 : 1, tiles = (double)B * H * Tk;
  const double per_key = rows == 1 ? 0.0292 : rows == 2 ? 0.0335 : rows <= 4 ? 0.0565 : 0.0745;
  const double here = width * per_key * Tk / kMaxSplits * (rows > 4 && heads > 8 ? 2.2 : 1);
  const double there = std::max(D <= 64 ? 29. : 43., 20 + width * 0.93e-3 * tiles) + 1.2e-3 * Tk / ((double)B * H);
  return here <= there;
}

int launch_attention_few(const AttentionArgs& a, bool bf16, cudaStream_t st) {
  const int rows = a.Tq * (a.H / a.Hkv);
  // blocks of a cluster per key head: until the GPU has four blocks per multiprocessor, each with 64 keys at least
  const long long heads = (long long)a.B * a.Hkv;
  int splits = 1;
  while (splits < kMaxSplits && heads * splits * 2 <= 148 * 4 && a.Tk / (splits * 2) >= 64) splits *= 2;
  if (bf16) return a.D <= 64 ? launch_few<__nv_bfloat16, 8>(a, rows, splits, st) : launch_few<__nv_bfloat16, 16>(a, rows, splits, st);
  return a.D <= 64 ? launch_few<float, 16>(a, rows, splits, st) : launch_few<float, 32>(a, rows, splits, st);
}

}  // namespace gshard
