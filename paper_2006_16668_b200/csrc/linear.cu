// The linear operator: pre = x . w + bias, y = act(pre) + residual, and its backward pass: the projections of
// a Transformer layer (section 2.1), with what surrounds the matrix product folded into its epilogue.
//
//   x [n, K], w [K, cols], bias [cols] (float), residual, y, pre [n, cols]
//   backward: dpre = dy act'(pre),  dx = dpre . w^T,  dw = x^T . dpre,  dbias = sum over rows of dpre
//
// bf16: the matrix products run on the tcgen05 GEMMs of the expert FFN (CTA pairs from 129 rows on); the
// forward's epilogue adds the bias, keeps pre, activates and adds the residual on the fp32 accumulator.
// dpre is rounded to bf16 once, as the operand of both gradient products (exact with no activation or relu on 16-bit
// dy); dbias sums it before the rounding.  Small products, whose time is launches, take what the rounding left as a
// second plane and a second pass, which halves the error of dx and dw to that of their own rounding.
// A product whose output tiles run at once is one launch (linear_mid.cu); another one (deep contractions) with
// too few tiles for the multiprocessors is cut along the contraction into runs whose fp32 partial products a second
// kernel adds in order.  Measured under the power cap, as a program that keeps the GPU busy has it: 65536 x 8192 -> 1024
// with residual 915 to 1000 us (1.1 to 1.2 PFLOP/s, tensor pipe 88 % active; a short burst 733 to 800); backward of
// 30011 x 1024 -> 8192 with gelu 1080 to 1110 us (burst 926: dpre 245, bound by HBM, dx 336, dw 346).
// fp32: an fp32 value is the exact sum of three bf16 values (8 bits of its 24 each; from 2^-110 on, below it what bf16's
// smallest step 2^-133 leaves), so x . w is six bf16 products of such planes on the same GEMMs, accumulated in fp32,
// smallest first; the three products left out lie below 2^-24.
// That is six times the tensor work and three times the operand bytes, and still several times faster than fp32 FMA
// on the CUDA cores (4100 x 1024 x 4096: 195 to 200 us, 160 to 170 in a burst, against 1172 there).  Infinities and NaN
// in x, w or dy give NaN.
// A few rows stream w through the CUDA cores instead (linear_few.cu).
#include <algorithm>

#include "activation.cuh"
#include "checks.cuh"
#include "gemm_dispatch.cuh"
#include "linear.cuh"
#include "pack.cuh"
#include "plan.cuh"
#include "umma_epilogue.cuh"

namespace gshard {

namespace {

using umma_epi::kPasses3;
constexpr int kSms = 148;                    // multiprocessors of a B200: sizes the work split, not the grids

// The operator's epilogue on `splits` fp32 partial products of n4 float4 each, added in order.
template <typename TY>
__global__ void __launch_bounds__(256) linear_finish_kernel(const float4* __restrict__ partial, int splits, LinearEpilogue lin,
                                                            void* y, long long n4, int cols4) {
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n4; i += (long long)gridDim.x * 256) {
    float4 s = partial[i];
#pragma unroll 8
    for (int k = 1; k < splits; ++k) {
      const float4 v = partial[(long long)k * n4 + i];
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    linear_epilogue4<TY>(lin, y, 4 * i, (int)(i % cols4) * 4, s);
  }
}

// Two tensors in one launch (the second may have no elements), n8 packs of 8 values each.
__global__ void __launch_bounds__(256) linear_split_kernel(const float* __restrict__ src0, __nv_bfloat16* __restrict__ dst0, long long n0,
                                                           const float* __restrict__ src1, __nv_bfloat16* __restrict__ dst1, long long n1) {
  for (long long at = (long long)blockIdx.x * 256 + threadIdx.x; at < n0 + n1; at += (long long)gridDim.x * 256) {
    const bool second = at >= n0;
    const float* src = second ? src1 : src0;
    __nv_bfloat16* dst = second ? dst1 : dst0;
    const long long n8 = second ? n1 : n0, i = second ? at - n0 : at;
    float f[8], hi[8], mid[8], lo[8];
    load_pack<float, 4>(src + 8 * i, f);
    load_pack<float, 4>(src + 8 * i + 4, f + 4);
    split3(f, hi, mid, lo, 8);
    store_pack<__nv_bfloat16, 8>(dst + 8 * i, hi);
    store_pack<__nv_bfloat16, 8>(dst + 8 * (n8 + i), mid);
    store_pack<__nv_bfloat16, 8>(dst + 8 * (2 * n8 + i), lo);
  }
}

// dpre = dy act'(pre) rounded to bf16 (where wanted), and the chunk's column sums of dpre before the rounding.
// A block covers 32 x 8 columns and one chunk of rows; a thread owns 8 columns and every 8th row, four of
// them in flight: the pass is bound by HBM (dy and pre in, dpre out).  PLANES: bf16 planes that dpre is
// written as: 3 (fp32), 2 (rounded, and what the rounding left) or 1.  Also clears the status word for the products that follow.
template <typename TY, int PLANES, int ACT>
__global__ void __launch_bounds__(256) linear_dpre_kernel(const TY* __restrict__ dy, const TY* __restrict__ pre, __nv_bfloat16* dpre,
                                                          float* __restrict__ partial, int* status, long long n, int cols, int chunk) {
  constexpr bool FAST = PLANES < 3;
  constexpr int U = sizeof(TY) == 2 ? 4 : 2;              // rows in flight
  constexpr int PW = 16 / (int)sizeof(TY), PN = 8 / PW;    // packs of 16 bytes per 8 columns
  __shared__ float part[8][256 + 8];
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
  if (threadIdx.x == 0 && blockIdx.x == 0 && blockIdx.y == 0) *status = 0;
  const int col = blockIdx.x * 256 + tx * 8;
  const long long r1 = min(n, (long long)(blockIdx.y + 1) * chunk);
  float sum[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) sum[j] = 0.f;
  if (col < cols) {
    for (long long r0 = (long long)blockIdx.y * chunk + ty; r0 < r1; r0 += 8 * U) {
      Pack<TY, PW> g[U][PN], v[U][PN];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (r0 + 8 * u < r1) {
          const long long off = (r0 + 8 * u) * cols + col;
#pragma unroll
          for (int h = 0; h < PN; ++h) {
            g[u][h].load_once(dy + off + h * PW);
            if (ACT != GSHARD_ACT_NONE) v[u][h].load_once(pre + off + h * PW);
          }
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (r0 + 8 * u < r1) {
          float d[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            d[j] = g[u][j / PW].get(j % PW);
            if (ACT != GSHARD_ACT_NONE) {
              const float a = v[u][j / PW].get(j % PW);
              // rounded before it is summed, whether or not it is also stored: the same bits for any set of outputs
              d[j] = __fmul_rn(d[j], FAST ? activation_slope_fast(a, ACT) : activation_slope(a, ACT));
            }
            sum[j] += d[j];
          }
          if (dpre) {
            const long long off = (r0 + 8 * u) * cols + col;
            if (PLANES == 2) {
              float hi[8], lo[8];
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                hi[j] = __bfloat162float(__float2bfloat16_rn(d[j]));
                lo[j] = fabsf(hi[j]) == INFINITY ? 0.f : d[j] - hi[j];     // an infinity is all in the first plane
              }
              store_pack<__nv_bfloat16, 8>(dpre + off, hi);
              store_pack<__nv_bfloat16, 8>(dpre + n * cols + off, lo);
            } else if (PLANES == 3) {
              float hi[8], mid[8], lo[8];
              split3(d, hi, mid, lo, 8);
              store_pack<__nv_bfloat16, 8>(dpre + off, hi);
              store_pack<__nv_bfloat16, 8>(dpre + n * cols + off, mid);
              store_pack<__nv_bfloat16, 8>(dpre + 2 * n * cols + off, lo);
            } else {
              store_pack<__nv_bfloat16, 8>(dpre + off, d);
            }
          }
        }
      }
    }
  }
  if (!partial) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) part[ty][tx * 8 + j] = sum[j];
  __syncthreads();
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c < cols) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += part[i][threadIdx.x];
    partial[(long long)blockIdx.y * cols + c] = s;
  }
}

template <typename TY, int PLANES>
void launch_dpre(const void* dy, const void* pre, void* dpre, float* partial, int* status, long long n, int cols, int chunk, int chunks, int act,
                 cudaStream_t st) {
  const dim3 grid(ceil_div(cols, 256), chunks);
#define GSHARD_DPRE(A)                                                                                                   \
  case A:                                                                                                                \
    linear_dpre_kernel<TY, PLANES, A><<<grid, 256, 0, st>>>(static_cast<const TY*>(dy), static_cast<const TY*>(pre),     \
                                                            static_cast<__nv_bfloat16*>(dpre), partial, status, n, cols, chunk); \
    break;
  switch (act) {
    GSHARD_DPRE(GSHARD_ACT_NONE)
    GSHARD_DPRE(GSHARD_ACT_RELU)
    GSHARD_DPRE(GSHARD_ACT_GELU)
    GSHARD_DPRE(GSHARD_ACT_GELU_TANH)
    GSHARD_DPRE(GSHARD_ACT_SILU)
  }
#undef GSHARD_DPRE
  count_launch();
}

// out[c] = sum over the partial rows: 8 strands of rows in order, then the strands.
__global__ void __launch_bounds__(256) linear_dbias_kernel(const float* __restrict__ partial, float* __restrict__ out, int rows,
                                                           int cols) {
  __shared__ float part[8][33];
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + tx;
  float s = 0.f;
  if (c < cols)
    for (int r = ty; r < rows; r += 8) s += partial[(long long)r * cols + c];
  part[ty][tx] = s;
  __syncthreads();
  if (ty == 0 && c < cols) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += part[i][tx];
    out[c] = s;
  }
}

int stride_grid(long long items) {
  return (int)std::max<long long>(1, std::min<long long>((items + 255) / 256, (long long)kSms * 16));
}

// Runs that a product [rows, cols] over `depth` is cut into: as many as fill the multiprocessors where the
// output has at most half as many tiles, each with at least four 64-deep k-blocks.
int splits_for(long long rows, int cols, long long depth) {
  const bool pairs = rows > 128;
  const long long tiles = pairs ? ((rows + 255) / 256) * ((cols + 255) / 256) : (cols + 255) / 256;
  const long long units = pairs ? kSms / 2 : kSms;
  const long long k_blocks = (depth + 63) / 64;
  if (tiles * 2 > units || k_blocks < 8) return 1;
  const long long s = std::min<long long>(units / tiles, k_blocks / 4);
  const long long per = (k_blocks + s - 1) / s;
  return (int)((k_blocks + per - 1) / per);      // no empty run at the end
}

// Whether w streams through the CUDA cores (linear_few.cu): up to 2 rows, and up to 8 of fp32 (whose planes would
// first be written) or where a product is not one launch of linear_mid.cu.  Measured, us, few to mid: 1024 -> 8192 6.8 to 7.5 for two rows, 8.2 to 7.6 for three, 10.5 to 7.5 for
// eight; 2048 -> 2048 5.9 to 6.5, 6.6 to 6.5, 8.8 to 6.5; 8192 -> 1024 8.0 to 9.8, 9.2 to 9.8, 11.6 to 9.8.
bool few_rows(int64_t n, bool bf16, MidShape mid) { return n <= 2 || (n <= 8 && !(bf16 && mid.bn)); }

}  // namespace

LinearPlan linear_plan(int64_t n, int K, int cols, int dtype, int out_dtype, bool backward) {
  Carver c;
  LinearPlan p{};
  const bool bf16 = dtype == GSHARD_BF16;
  p.status = c.take(256);
  if (!backward) p.mid = linear_mid_shape(n, cols, K, bf16 ? 1 : kPasses3, out_dtype == GSHARD_F32);
  if (n == 0 || (!backward && few_rows(n, bf16, p.mid))) { p.total = c.off; return p; }
  p.xp = c.take(bf16 ? 0 : (size_t)n * K * 6);             // planes of fp32 operands
  p.wp = c.take(bf16 ? 0 : (size_t)K * cols * 6);
  if (!backward) {
    p.splits = p.mid.bn ? 1 : splits_for(n, cols, K);
    if (p.splits > 1) p.join = c.take((size_t)p.splits * n * cols * 4);
    p.total = c.off;
    return p;
  }
  // a second pass of a product below 2^32 operations takes at most about 3 us
  p.planes = !bf16 ? 3 : 2.0 * n * K * cols <= 4294967296.0 ? 2 : 1;
  p.dpre = c.take((size_t)n * cols * 2 * p.planes);
  const int col_blocks = ceil_div(cols, 256);
  const long long want = std::max(1, kSms * 8 / col_blocks);                // row chunks that give every multiprocessor 8 blocks
  p.chunk = (int)std::max<long long>(32, (n + want - 1) / want);
  p.chunks = (int)((n + p.chunk - 1) / p.chunk);
  p.colsum = c.take((size_t)p.chunks * cols * 4);
  p.dx_mid = linear_mid_shape(n, K, cols, bf16 ? p.planes : kPasses3, !bf16);
  p.dw_mid = linear_mid_shape(K, cols, n, bf16 ? p.planes : kPasses3, !bf16);
  p.dx_splits = p.dx_mid.bn ? 1 : splits_for(n, K, cols);
  p.dw_splits = p.dw_mid.bn ? 1 : splits_for(K, cols, n);
  p.join = c.take(std::max(p.dx_splits > 1 ? (size_t)p.dx_splits * n * K * 4 : 0,
                           p.dw_splits > 1 ? (size_t)p.dw_splits * K * cols * 4 : 0));
  p.total = c.off;
  return p;
}

int linear_validate(int64_t n, int32_t K, int32_t cols, int32_t dtype, int32_t out_dtype) {
  if (n < 0 || K <= 0 || cols <= 0) return GSHARD_ERR_INVALID_ARG;
  if (dtype != GSHARD_F32 && dtype != GSHARD_BF16) return GSHARD_ERR_INVALID_ARG;
  if (out_dtype != GSHARD_F32 && out_dtype != dtype) return GSHARD_ERR_INVALID_ARG;
  if (K % 8 || cols % 8 || K > (1 << 24) || cols > (1 << 24)) return GSHARD_ERR_UNSUPPORTED_SHAPE;
  // a tensor map's strides; tile counts in 31 bits
  if (n > (1ll << 30) || n * std::max(K, cols) >= (1ll << 37) || (long long)K * cols >= (1ll << 37)) return GSHARD_ERR_UNSUPPORTED_SHAPE;
  if (((std::max<long long>(n, K) + 127) / 128) * ((long long)(std::max(K, cols) + 127) / 128) >= (1ll << 30)) return GSHARD_ERR_UNSUPPORTED_SHAPE;
  return GSHARD_OK;
}

void linear_split_planes(const void* src0, void* dst0, long long n0, const void* src1, void* dst1, long long n1, cudaStream_t st) {
  linear_split_kernel<<<stride_grid((n0 + n1) / 8), 256, 0, st>>>(static_cast<const float*>(src0), static_cast<__nv_bfloat16*>(dst0), n0 / 8,
                                                                  static_cast<const float*>(src1), static_cast<__nv_bfloat16*>(dst1), n1 / 8);
  count_launch();
}

namespace {

// the tensor-core GEMMs, whose operands are bf16 (or planes of it)
Dims linear_dims(int K, int cols) {
  gshard_moe_shape one{};
  one.G = 1; one.S = 1; one.C = 1; one.E = 2; one.M = K; one.H = cols; one.dtype = GSHARD_BF16;
  return make_dims(one);
}
// C = A . B: in one launch of linear_mid.cu, or cut into `splits` runs through the fp32 partial products in `join`
int gemm_joined(const Dims& d, UmmaGemm g, MidShape mid, int splits, float* join, int* status, cudaStream_t st) {
  const LinearEpilogue none{};
  if (mid.bn) return launch_linear_mid(g, none, mid, g.clear_status != 0, status, st);
  if (g.planes_a == 3) { g.linear = &none; g.runs = 1; }
  if (splits <= 1) return run_gemm(d, g, status, st);
  void* out = g.C;
  const bool out_f32 = g.out_f32 != 0;
  const long long n4 = (long long)g.rows * g.cols / 4;
  g.C = join; g.out_f32 = 1; g.splits = splits; g.c_bs = (long long)g.rows * g.cols;
  GS_CHECK(run_gemm(d, g, status, st));
  const float4* partial = reinterpret_cast<const float4*>(join);
  if (out_f32) linear_finish_kernel<float><<<stride_grid(n4), 256, 0, st>>>(partial, splits, none, out, n4, g.cols / 4);
  else linear_finish_kernel<__nv_bfloat16><<<stride_grid(n4), 256, 0, st>>>(partial, splits, none, out, n4, g.cols / 4);
  count_launch();
  return GSHARD_OK;
}

int zero(void* p, size_t bytes, cudaStream_t st) {
  if (!p || cudaMemsetAsync(p, 0, bytes, st) == cudaSuccess) return GSHARD_OK;
  cudaGetLastError();
  return GSHARD_ERR_CUDA;
}

}  // namespace

int linear_run_forward(int64_t n_rows, int K, int cols, int dtype, int out_dtype, const LinearEpilogue& lin, const void* x,
                       const void* w, void* y, const LinearPlan& pl, unsigned char* ws, cudaStream_t st) {
  int* status = reinterpret_cast<int*>(ws);
  const bool out_f32 = out_dtype == GSHARD_F32;
  if (few_rows(n_rows, dtype == GSHARD_BF16, pl.mid)) {
    GS_CHECK(launch_linear_few((int)n_rows, K, cols, dtype == GSHARD_BF16, out_f32, x, w, y, lin, status, st));
    return cudaGetLastError() == cudaSuccess ? GSHARD_OK : GSHARD_ERR_CUDA;
  }
  const Dims d = linear_dims(K, cols);
  UmmaGemm g{};
  g.A = x; g.B = w; g.C = y; g.rows = (int)n_rows; g.cols = cols; g.K = K; g.batch = 1;
  g.a_kmajor = true; g.b_kmajor = false; g.a_ld = K; g.b_ld = cols; g.c_ld = cols;
  g.clear_status = 1;
  g.a_stream = 1; g.prefer_two_sm = 1; g.out_f32 = out_f32;
  if (dtype == GSHARD_F32) {
    linear_split_planes(x, ws + pl.xp, n_rows * K, w, ws + pl.wp, (long long)K * cols, st);
    g.A = ws + pl.xp; g.B = ws + pl.wp; g.planes_a = g.planes_b = 3; g.a_bs = n_rows * K; g.b_bs = (long long)K * cols; g.a_stream = 0;
  }
  if (pl.mid.bn) return launch_linear_mid(g, lin, pl.mid, true, status, st);
  g.runs = out_f32;
  if (pl.splits == 1) {
    g.linear = &lin;
    GS_CHECK(run_gemm(d, g, status, st));
  } else {
    const long long n4 = n_rows * cols / 4;
    const LinearEpilogue none{};
    if (g.runs) g.linear = &none;
    g.C = ws + pl.join; g.out_f32 = 1; g.splits = pl.splits; g.c_bs = n_rows * cols;
    GS_CHECK(run_gemm(d, g, status, st));
    const float4* partial = reinterpret_cast<const float4*>(ws + pl.join);
    if (out_f32) linear_finish_kernel<float><<<stride_grid(n4), 256, 0, st>>>(partial, pl.splits, lin, y, n4, cols / 4);
    else linear_finish_kernel<__nv_bfloat16><<<stride_grid(n4), 256, 0, st>>>(partial, pl.splits, lin, y, n4, cols / 4);
    count_launch();
  }
  return cudaGetLastError() == cudaSuccess ? GSHARD_OK : GSHARD_ERR_CUDA;
}

int linear_run_gradients(int64_t n_rows, int K, int cols, bool fp32, int planes, const void* x, const void* w, const void* dpre, void* dx,
                         void* dw, const LinearPlan& pl, unsigned char* ws, bool cleared, cudaStream_t st) {
  int* status = reinterpret_cast<int*>(ws);
  const Dims d = linear_dims(K, cols);
  float* join = reinterpret_cast<float*>(ws + pl.join);
  if (fp32 && (dx || dw))
    linear_split_planes(w, ws + pl.wp, dx ? (long long)K * cols : 0, x, ws + pl.xp, dw ? n_rows * K : 0, st);
  if (dx) {                                       // [n, K] = dpre [n, cols] . w^T, both contiguous along cols
    UmmaGemm g{};
    g.A = dpre; g.B = w; g.C = dx; g.rows = (int)n_rows; g.cols = K; g.K = cols; g.batch = 1;
    g.a_kmajor = true; g.b_kmajor = true; g.a_ld = cols; g.b_ld = cols; g.c_ld = K;
    g.prefer_two_sm = 1; g.out_f32 = fp32; g.clear_status = !cleared;
    cleared = true;
    if (fp32) {
      g.B = ws + pl.wp; g.planes_a = g.planes_b = 3; g.a_bs = n_rows * cols; g.b_bs = (long long)K * cols;
    } else if (planes == 2) {
      g.planes_a = 2; g.planes_b = 1; g.a_bs = n_rows * cols;
    }
    GS_CHECK(gemm_joined(d, g, pl.dx_mid, pl.dx_splits, join, status, st));
  }
  if (dw) {                                       // [K, cols] = x^T . dpre, both stored row by row of the contraction
    UmmaGemm g{};
    g.A = x; g.B = dpre; g.C = dw; g.rows = K; g.cols = cols; g.K = (int)n_rows; g.batch = 1;
    g.a_kmajor = false; g.b_kmajor = false; g.a_ld = K; g.b_ld = cols; g.c_ld = cols;
    g.prefer_two_sm = 1; g.out_f32 = fp32; g.clear_status = !cleared;
    if (fp32) {
      g.A = ws + pl.xp; g.planes_a = g.planes_b = 3; g.a_bs = n_rows * K; g.b_bs = n_rows * cols;
    } else if (planes == 2) {
      g.planes_a = 1; g.planes_b = 2; g.b_bs = n_rows * cols;
    }
    GS_CHECK(gemm_joined(d, g, pl.dw_mid, pl.dw_splits, join, status, st));
  }
  return cudaGetLastError() == cudaSuccess ? GSHARD_OK : GSHARD_ERR_CUDA;
}

}  // namespace gshard

using namespace gshard;

extern "C" {

size_t gshard_linear_workspace_bytes(int64_t n_rows, int32_t K, int32_t cols, int32_t dtype, int32_t out_dtype, int for_backward) {
  if (linear_validate(n_rows, K, cols, dtype, out_dtype) != GSHARD_OK) return 0;
  return linear_plan(n_rows, K, cols, dtype, out_dtype, for_backward != 0).total;
}

int gshard_linear_forward(int64_t n_rows, int32_t K, int32_t cols, int32_t dtype, int32_t out_dtype, int32_t activation,
                          const void* x, const void* w, const float* bias, const void* residual, void* y, void* pre,
                          void* workspace, size_t workspace_bytes, void* cuda_stream) {
  launch_counter().n = 0;
  GS_CHECK(linear_validate(n_rows, K, cols, dtype, out_dtype));
  if (activation < GSHARD_ACT_NONE || activation > GSHARD_ACT_SILU) return GSHARD_ERR_INVALID_ARG;
  if (n_rows == 0) return GSHARD_OK;
  GS_CHECK_PTR(x); GS_CHECK_PTR(w); GS_CHECK_PTR(y);
  GS_CHECK_OPTIONAL_PTR(bias); GS_CHECK_OPTIONAL_PTR(residual); GS_CHECK_OPTIONAL_PTR(pre);
  if (y == x || y == w || pre == x || pre == w || (pre && (pre == y || pre == residual))) return GSHARD_ERR_INVALID_ARG;
  const LinearPlan pl = linear_plan(n_rows, K, cols, dtype, out_dtype, false);
  GS_CHECK_WORKSPACE(workspace, workspace_bytes, pl.total);
  GS_CHECK(check_device());
  NvtxRange range("gshard.linear");
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  return linear_run_forward(n_rows, K, cols, dtype, out_dtype, LinearEpilogue{bias, residual, pre, activation}, x, w, y, pl,
                            static_cast<unsigned char*>(workspace), st);
}

int gshard_linear_backward(int64_t n_rows, int32_t K, int32_t cols, int32_t dtype, int32_t out_dtype, int32_t activation,
                           const void* x, const void* w, const void* pre, const void* dy, void* dx, void* dw, float* dbias,
                           void* workspace, size_t workspace_bytes, void* cuda_stream) {
  launch_counter().n = 0;
  GS_CHECK(linear_validate(n_rows, K, cols, dtype, out_dtype));
  if (activation < GSHARD_ACT_NONE || activation > GSHARD_ACT_SILU) return GSHARD_ERR_INVALID_ARG;
  const size_t es = dtype == GSHARD_BF16 ? 2 : 4;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  GS_CHECK_OPTIONAL_PTR(dx); GS_CHECK_OPTIONAL_PTR(dw); GS_CHECK_OPTIONAL_PTR(dbias);
  // two gradients in one place (n_rows == K, K == cols or a single row make their sizes agree)
  if ((dx && dx == dw) || (dbias && (dbias == dx || dbias == dw))) return GSHARD_ERR_INVALID_ARG;
  if (n_rows == 0) {                              // no rows: the weight gradients are empty sums
    if (!dw && !dbias) return GSHARD_OK;
    GS_CHECK(check_device());
    GS_CHECK(zero(dw, (size_t)K * cols * es, st));
    return zero(dbias, (size_t)cols * 4, st);
  }
  GS_CHECK_PTR(dy);
  if (dx) GS_CHECK_PTR(w);
  if (dw) GS_CHECK_PTR(x);
  if (activation != GSHARD_ACT_NONE) GS_CHECK_PTR(pre);
  if (dx && (dx == dy || dx == x || dx == w || dx == pre)) return GSHARD_ERR_INVALID_ARG;
  if (dw && (dw == dy || dw == x || dw == w || dw == pre)) return GSHARD_ERR_INVALID_ARG;
  const LinearPlan pl = linear_plan(n_rows, K, cols, dtype, out_dtype, true);
  GS_CHECK_WORKSPACE(workspace, workspace_bytes, pl.total);
  GS_CHECK(check_device());
  NvtxRange range("gshard.linear.backward");
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  int* status = reinterpret_cast<int*>(ws);
  if (!dx && !dw && !dbias) return zero(status, sizeof(int), st);
  const bool fp32 = dtype == GSHARD_F32;
  const bool convert = fp32 || activation != GSHARD_ACT_NONE || out_dtype != dtype;    // else dpre is dy itself
  // dy times 0 or 1 needs no second plane
  const bool exact = out_dtype == dtype && (activation == GSHARD_ACT_NONE || activation == GSHARD_ACT_RELU);
  const int planes = !fp32 && exact ? 1 : pl.planes;
  void* buf = convert && (dx || dw) ? ws + pl.dpre : nullptr;
  float* colsum = dbias ? reinterpret_cast<float*>(ws + pl.colsum) : nullptr;
  if (buf || colsum) {
#define GSHARD_DPRE(TY, P) launch_dpre<TY, P>(dy, pre, buf, colsum, status, n_rows, cols, pl.chunk, pl.chunks, activation, st)
    if (planes == 3) GSHARD_DPRE(float, 3);
    else if (out_dtype == GSHARD_F32) { if (planes == 2) GSHARD_DPRE(float, 2); else GSHARD_DPRE(float, 1); }
    else { if (planes == 2) GSHARD_DPRE(__nv_bfloat16, 2); else GSHARD_DPRE(__nv_bfloat16, 1); }
#undef GSHARD_DPRE
    if (dbias) {
      linear_dbias_kernel<<<ceil_div(cols, 32), 256, 0, st>>>(colsum, dbias, pl.chunks, cols);
      count_launch();
    }
  }
  const void* dpre = convert ? buf : dy;
  const bool cleared = buf || colsum;             // the status word, by the first kernel of the call
  return linear_run_gradients(n_rows, K, cols, fp32, planes, x, w, dpre, dx, dw, pl, ws, cleared, st);
}

}  // extern "C"
