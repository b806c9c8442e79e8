// The linear operator: pre = x . w + bias, y = act(pre) + residual, and its backward pass: the projections of
// a Transformer layer (section 2.1), with what surrounds the matrix product folded into its epilogue.
//
//   x [n, K], w [K, cols], bias [cols] (float), residual, y, pre [n, cols]
//   backward: dpre = dy act'(pre),  dx = dpre . w^T,  dw = x^T . dpre,  dbias = sum over rows of dpre
//
// bf16: the matrix products run on the tcgen05 GEMMs of the expert FFN (CTA pairs from 129 rows on); the
// forward's epilogue adds the bias, keeps pre, activates and adds the residual on the fp32 accumulator.
// dpre is rounded to bf16 once, as the operand of both gradient products; dbias sums it before the rounding.
// A product with too few output tiles for the multiprocessors is cut along the contraction into runs whose
// fp32 partial products a second kernel adds in order.
// fp32: CUDA cores, fp32 FMA.
#include <algorithm>

#include "activation.cuh"
#include "checks.cuh"
#include "gemm_dispatch.cuh"
#include "pack.cuh"
#include "plan.cuh"

namespace gshard {

namespace {

constexpr int kSms = 148;                    // multiprocessors of a B200: sizes the work split, not the grids

// The rest of the operator on the fp32 product x . w.
__global__ void __launch_bounds__(256) linear_finish_kernel(const float* __restrict__ product, float* y,
                                                            const float* __restrict__ bias, const float* residual,
                                                            float* pre, long long n4, int cols4, int act) {
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n4; i += (long long)gridDim.x * 256) {
    const float4 v = reinterpret_cast<const float4*>(product)[i];
    float f[4] = {v.x, v.y, v.z, v.w};
    if (bias) {
      const float4 b = __ldg(reinterpret_cast<const float4*>(bias) + i % cols4);
      f[0] += b.x; f[1] += b.y; f[2] += b.z; f[3] += b.w;
    }
    if (pre) reinterpret_cast<float4*>(pre)[i] = make_float4(f[0], f[1], f[2], f[3]);
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = activation_value(f[j], act);
    if (residual) {
      const float4 r = reinterpret_cast<const float4*>(residual)[i];
      f[0] += r.x; f[1] += r.y; f[2] += r.z; f[3] += r.w;
    }
    reinterpret_cast<float4*>(y)[i] = make_float4(f[0], f[1], f[2], f[3]);
  }
}

// dpre = dy act'(pre) rounded to TD (where wanted), and the chunk's column sums of dpre before the rounding.
// A block covers 32 x 8 columns and one chunk of rows; a thread owns 8 columns and every 8th row, four of
// them in flight: the pass is bound by HBM (dy and pre in, dpre out).
template <typename TY, typename TD, int ACT>
__global__ void __launch_bounds__(256) linear_dpre_kernel(const TY* __restrict__ dy, const TY* __restrict__ pre, TD* dpre,
                                                          float* __restrict__ partial, long long n, int cols, int chunk) {
  constexpr bool FAST = sizeof(TD) == 2;
  constexpr int U = sizeof(TY) == 2 ? 4 : 2;              // rows in flight
  constexpr int PW = 16 / (int)sizeof(TY), PN = 8 / PW;    // packs of 16 bytes per 8 columns
  __shared__ float part[8][256 + 8];
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
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
#pragma unroll
            for (int h = 0; h < 8; h += 16 / (int)sizeof(TD)) store_pack<TD, 16 / (int)sizeof(TD)>(dpre + off + h, d + h);
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

template <typename TY, typename TD>
void launch_dpre(const void* dy, const void* pre, void* dpre, float* partial, long long n, int cols, int chunk, int chunks, int act,
                 cudaStream_t st) {
  const dim3 grid(ceil_div(cols, 256), chunks);
#define GSHARD_DPRE(A)                                                                                                   \
  case A:                                                                                                                \
    linear_dpre_kernel<TY, TD, A><<<grid, 256, 0, st>>>(static_cast<const TY*>(dy), static_cast<const TY*>(pre),         \
                                                        static_cast<TD*>(dpre), partial, n, cols, chunk);                \
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

// out = sum of `splits` fp32 partial products of n4 float4 each, in order, rounded to bf16.
__global__ void __launch_bounds__(256) linear_join_kernel(const float4* __restrict__ partial, uint2* __restrict__ out,
                                                          long long n4, int splits) {
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n4; i += (long long)gridDim.x * 256) {
    float4 s = partial[i];
    for (int k = 1; k < splits; ++k) {
      const float4 v = partial[(long long)k * n4 + i];
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    const __nv_bfloat162 a = __floats2bfloat162_rn(s.x, s.y), b = __floats2bfloat162_rn(s.z, s.w);
    out[i] = make_uint2(*reinterpret_cast<const unsigned*>(&a), *reinterpret_cast<const unsigned*>(&b));
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

struct LinearPlan { size_t status, dpre, colsum, join, total; int chunks, chunk, dx_splits, dw_splits; };

LinearPlan linear_plan(int64_t n, int K, int cols, int dtype, bool backward) {
  Carver c;
  LinearPlan p{};
  const bool bf16 = dtype == GSHARD_BF16;
  p.status = c.take(256);
  if (!backward && !bf16) p.join = c.take((size_t)n * cols * 4);           // the product before its epilogue
  if (!backward || n == 0) { p.total = c.off; return p; }
  p.dpre = c.take((size_t)n * cols * (bf16 ? 2 : 4));
  const int col_blocks = ceil_div(cols, 256);
  const long long want = std::max(1, kSms * 8 / col_blocks);                // row chunks that give every multiprocessor 8 blocks
  p.chunk = (int)std::max<long long>(32, (n + want - 1) / want);
  p.chunks = (int)((n + p.chunk - 1) / p.chunk);
  p.colsum = c.take((size_t)p.chunks * cols * 4);
  p.dx_splits = bf16 ? splits_for(n, K, cols) : 1;
  p.dw_splits = bf16 ? splits_for(K, cols, n) : 1;
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
  // 64-row tiles of the CUDA-core GEMM in a grid's y extent; a tensor map's strides; tile counts in 31 bits
  if (dtype == GSHARD_F32 && ((n + 63) / 64 > 65535 || (K + 63) / 64 > 65535)) return GSHARD_ERR_UNSUPPORTED_SHAPE;
  if (n > (1ll << 30) || n * std::max(K, cols) >= (1ll << 37)) return GSHARD_ERR_UNSUPPORTED_SHAPE;
  if (((n + 127) / 128) * ((long long)(std::max(K, cols) + 127) / 128) >= (1ll << 30)) return GSHARD_ERR_UNSUPPORTED_SHAPE;
  return GSHARD_OK;
}

Dims linear_dims(int K, int cols, int dtype) {
  gshard_moe_shape one{};
  one.G = 1; one.S = 1; one.C = 1; one.E = 2; one.M = K; one.H = cols; one.dtype = dtype;
  return make_dims(one);
}

// C = A . B (bf16 out) cut into `splits` runs through the fp32 partial products in `join`
int gemm_joined(const Dims& d, UmmaGemm g, int splits, float* join, int* status, cudaStream_t st) {
  if (splits <= 1) return run_gemm(d, g, status, st);
  void* out = g.C;
  const long long n4 = (long long)g.rows * g.cols / 4;
  g.C = join; g.out_f32 = 1; g.splits = splits; g.c_bs = (long long)g.rows * g.cols;
  GS_CHECK(run_gemm(d, g, status, st));
  linear_join_kernel<<<stride_grid(n4), 256, 0, st>>>(reinterpret_cast<const float4*>(join), static_cast<uint2*>(out), n4, splits);
  count_launch();
  return GSHARD_OK;
}

int zero(void* p, size_t bytes, cudaStream_t st) {
  if (!p || cudaMemsetAsync(p, 0, bytes, st) == cudaSuccess) return GSHARD_OK;
  cudaGetLastError();
  return GSHARD_ERR_CUDA;
}

}  // namespace

}  // namespace gshard

using namespace gshard;

extern "C" {

size_t gshard_linear_workspace_bytes(int64_t n_rows, int32_t K, int32_t cols, int32_t dtype, int32_t out_dtype, int for_backward) {
  if (linear_validate(n_rows, K, cols, dtype, out_dtype) != GSHARD_OK) return 0;
  return linear_plan(n_rows, K, cols, dtype, for_backward != 0).total;
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
  const LinearPlan pl = linear_plan(n_rows, K, cols, dtype, false);
  GS_CHECK_WORKSPACE(workspace, workspace_bytes, pl.total);
  GS_CHECK(check_device());
  NvtxRange range("gshard.linear");
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  int* status = static_cast<int*>(workspace);
  GS_CHECK(zero(status, sizeof(int), st));
  const Dims d = linear_dims(K, cols, dtype);
  UmmaGemm g{};
  g.A = x; g.B = w; g.C = y; g.rows = (int)n_rows; g.cols = cols; g.K = K; g.batch = 1;
  g.a_kmajor = true; g.b_kmajor = false; g.a_ld = K; g.b_ld = cols; g.c_ld = cols;
  g.a_stream = 1; g.prefer_two_sm = 1; g.out_f32 = out_dtype == GSHARD_F32;
  LinearEpilogue lin{bias, residual, pre, activation};
  if (dtype == GSHARD_BF16) {
    g.linear = &lin;
    GS_CHECK(run_gemm(d, g, status, st));
  } else {
    float* product = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + pl.join);
    g.C = product;
    GS_CHECK(run_gemm(d, g, status, st));
    const long long n4 = n_rows * cols / 4;
    linear_finish_kernel<<<stride_grid(n4), 256, 0, st>>>(product, static_cast<float*>(y), bias,
                                                          static_cast<const float*>(residual), static_cast<float*>(pre), n4,
                                                          cols / 4, activation);
    count_launch();
  }
  return cudaGetLastError() == cudaSuccess ? GSHARD_OK : GSHARD_ERR_CUDA;
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
  const LinearPlan pl = linear_plan(n_rows, K, cols, dtype, true);
  GS_CHECK_WORKSPACE(workspace, workspace_bytes, pl.total);
  GS_CHECK(check_device());
  NvtxRange range("gshard.linear.backward");
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  int* status = reinterpret_cast<int*>(ws);
  GS_CHECK(zero(status, sizeof(int), st));
  const bool convert = activation != GSHARD_ACT_NONE || out_dtype != dtype;    // else dpre is dy itself
  void* buf = convert && (dx || dw) ? ws + pl.dpre : nullptr;
  float* colsum = dbias ? reinterpret_cast<float*>(ws + pl.colsum) : nullptr;
  if (buf || colsum) {
    if (dtype == GSHARD_F32) launch_dpre<float, float>(dy, pre, buf, colsum, n_rows, cols, pl.chunk, pl.chunks, activation, st);
    else if (out_dtype == GSHARD_F32) launch_dpre<float, __nv_bfloat16>(dy, pre, buf, colsum, n_rows, cols, pl.chunk, pl.chunks, activation, st);
    else launch_dpre<__nv_bfloat16, __nv_bfloat16>(dy, pre, buf, colsum, n_rows, cols, pl.chunk, pl.chunks, activation, st);
    if (dbias) {
      linear_dbias_kernel<<<ceil_div(cols, 32), 256, 0, st>>>(colsum, dbias, pl.chunks, cols);
      count_launch();
    }
  }
  const void* dpre = convert ? buf : dy;
  const Dims d = linear_dims(K, cols, dtype);
  float* join = reinterpret_cast<float*>(ws + pl.join);
  if (dx) {                                       // [n, K] = dpre [n, cols] . w^T, both contiguous along cols
    UmmaGemm g{};
    g.A = dpre; g.B = w; g.C = dx; g.rows = (int)n_rows; g.cols = K; g.K = cols; g.batch = 1;
    g.a_kmajor = true; g.b_kmajor = true; g.a_ld = cols; g.b_ld = cols; g.c_ld = K;
    g.prefer_two_sm = 1;
    GS_CHECK(gemm_joined(d, g, pl.dx_splits, join, status, st));
  }
  if (dw) {                                       // [K, cols] = x^T . dpre, both stored row by row of the contraction
    UmmaGemm g{};
    g.A = x; g.B = dpre; g.C = dw; g.rows = K; g.cols = cols; g.K = (int)n_rows; g.batch = 1;
    g.a_kmajor = false; g.b_kmajor = false; g.a_ld = K; g.b_ld = cols; g.c_ld = cols;
    g.prefer_two_sm = 1;
    GS_CHECK(gemm_joined(d, g, pl.dw_splits, join, status, st));
  }
  return cudaGetLastError() == cudaSuccess ? GSHARD_OK : GSHARD_ERR_CUDA;
}

}  // extern "C"
