// Layer norm over the last dimension of x [n, M], the normalisation that follows the residual
// connection of every sub-layer (section 2.1), and its backward pass.
//
//   mu = mean(x), r = 1 / sqrt(mean((x - mu)^2) + eps), z = (x - mu) r, y = gamma z + beta
//   backward: g = gamma dy,  dx = r (g - mean(g) - z mean(g z)) [+ dskip]
//             dgamma = sum over rows of dy z,  dbeta = sum over rows of dy
//
// Both passes are bound by HBM: x is read and y written once, and a row lives in the registers of the
// threads that own it ("a team": one warp up to 1024 elements, up to 32 warps beyond), so that the
// mean, the variance about that mean and the normalisation need no second pass over memory.  All sums
// are fp32; the only rounding to 16 bits is the one of the stored y and dx.
// The weight gradients are sums over rows: a team keeps its columns' share in registers over all the
// rows it walks, a block writes one partial row, and a second kernel adds the partial rows in a fixed
// order, so that the result has the same bits from run to run.
#include <algorithm>

#include "checks.cuh"
#include "pack.cuh"

namespace gshard {

namespace {

constexpr int kLnMaxTeam = 1024;
constexpr int kLnMaxM = 16 * kLnMaxTeam;
constexpr int kLnSms = 148;                  // multiprocessors of a B200; only sizes the partial rows

// W floats of a parameter vector (16-byte loads where W allows)
template <int W>
__device__ __forceinline__ void load_param(const float* p, float* f) {
  constexpr int C = W < 4 ? W : 4;
#pragma unroll
  for (int j = 0; j < W; j += C) load_pack<float, C>(p + j, f + j);
}

// Sums of K values over the team.  A team of one warp stays inside the warp; a larger team is the whole
// block.  `buf` holds 32 * K floats and is reused by the next call: callers alternate two of them.
template <int K>
__device__ __forceinline__ void team_sum(float (&s)[K], float* buf) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1)
#pragma unroll
    for (int k = 0; k < K; ++k) s[k] += __shfl_xor_sync(0xffffffffu, s[k], off);
  if (blockDim.x > 32) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    if (lane == 0)
#pragma unroll
      for (int k = 0; k < K; ++k) buf[k * 32 + warp] = s[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float t = lane < warps ? buf[k * 32 + lane] : 0.f;
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) t += __shfl_xor_sync(0xffffffffu, t, off);
      s[k] = t;
    }
  }
}

// NT: threads of the block at most (256: one-warp teams, else one team of the whole block).
template <typename T, int W, int VPT, int NT>
__global__ void __launch_bounds__(NT) ln_fwd_kernel(const T* __restrict__ x, const float* __restrict__ gamma, const float* __restrict__ beta,
                              T* y, float* __restrict__ mean, float* __restrict__ rstd, long long n, int M, float eps) {
  __shared__ float buf[2][32];
  const int packs = M / W;
  const float inv_m = 1.f / (float)M;
  for (long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y; row < n; row += (long long)gridDim.x * blockDim.y) {
    const T* xr = x + row * M;
    float v[VPT][W];
    float s[1] = {0.f};
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int p = i * blockDim.x + threadIdx.x;
      if (p < packs) {
        load_pack<T, W>(xr + (long long)p * W, v[i]);
      } else {
#pragma unroll
        for (int j = 0; j < W; ++j) v[i][j] = 0.f;
      }
    }
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int j = 0; j < W; ++j) s[0] += v[i][j];
    team_sum<1>(s, buf[0]);
    const float mu = s[0] * inv_m;
    float q[1] = {0.f};
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      if (i * (int)blockDim.x + (int)threadIdx.x < packs) {
#pragma unroll
        for (int j = 0; j < W; ++j) { v[i][j] -= mu; q[0] = fmaf(v[i][j], v[i][j], q[0]); }
      }
    }
    team_sum<1>(q, buf[1]);
    const float r = 1.f / sqrtf(q[0] * inv_m + eps);
    if (threadIdx.x == 0) {
      if (mean) mean[row] = mu;
      if (rstd) rstd[row] = r;
    }
    T* yr = y + row * M;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int p = i * blockDim.x + threadIdx.x;
      if (p < packs) {
        float gm[W], o[W];
        load_param<W>(gamma + (long long)p * W, gm);
#pragma unroll
        for (int j = 0; j < W; ++j) o[j] = v[i][j] * r * gm[j];
        if (beta) {
          float bt[W];
          load_param<W>(beta + (long long)p * W, bt);
#pragma unroll
          for (int j = 0; j < W; ++j) o[j] += bt[j];
        }
        store_pack<T, W>(yr + (long long)p * W, o);
      }
    }
  }
}

// Block b's share of the weight gradients goes to partial[b][0..M) (dgamma) and partial[b][M..2M) (dbeta).
// A thread's columns are summed in registers, or (SUMS_IN_SMEM, rows beyond 8192 elements, where the
// register file does not hold a row and its sums) in its own words of shared memory.
template <typename T, int W, int VPT, int NT, bool SUMS_IN_SMEM>
__global__ void __launch_bounds__(NT) ln_bwd_kernel(const T* __restrict__ x, const float* __restrict__ gamma, const float* __restrict__ mean,
                              const float* __restrict__ rstd, const T* dy, const T* dskip, T* dx, float* __restrict__ partial,
                              long long n, int M) {
  extern __shared__ float sums[];              // 2 M floats: several teams in the block, or SUMS_IN_SMEM
  __shared__ float buf[2][64];
  const int packs = M / W;
  const float inv_m = 1.f / (float)M;
  float ag[SUMS_IN_SMEM ? 1 : VPT][W], ab[SUMS_IN_SMEM ? 1 : VPT][W];
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int p = i * blockDim.x + threadIdx.x;
#pragma unroll
    for (int j = 0; j < W; ++j) {
      if (!SUMS_IN_SMEM) { ag[i][j] = 0.f; ab[i][j] = 0.f; }
      else if (partial && p < packs) { sums[j * packs + p] = 0.f; sums[M + j * packs + p] = 0.f; }
    }
  }
  int flip = 0;
  for (long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y; row < n; row += (long long)gridDim.x * blockDim.y) {
    const T* xr = x + row * M;
    const T* dyr = dy + row * M;
    const float mu = mean[row], r = rstd[row];
    float z[VPT][W], g[VPT][W];
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int p = i * blockDim.x + threadIdx.x;
      if (p < packs) {
        load_pack<T, W>(xr + (long long)p * W, z[i]);
        load_pack<T, W>(dyr + (long long)p * W, g[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int p = i * blockDim.x + threadIdx.x;
      if (p < packs) {
        float gm[W];
        load_param<W>(gamma + (long long)p * W, gm);
#pragma unroll
        for (int j = 0; j < W; ++j) {
          z[i][j] = (z[i][j] - mu) * r;
          if (SUMS_IN_SMEM) {
            if (partial) {
              sums[j * packs + p] = fmaf(g[i][j], z[i][j], sums[j * packs + p]);
              sums[M + j * packs + p] += g[i][j];
            }
          } else {
            ab[i][j] += g[i][j];
            ag[i][j] = fmaf(g[i][j], z[i][j], ag[i][j]);
          }
          g[i][j] *= gm[j];
          s[0] += g[i][j];
          s[1] = fmaf(g[i][j], z[i][j], s[1]);
        }
      }
    }
    team_sum<2>(s, buf[flip]);
    flip ^= 1;
    const float c0 = s[0] * inv_m, c1 = s[1] * inv_m;
    T* dxr = dx + row * M;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int p = i * blockDim.x + threadIdx.x;
      if (p < packs) {
        float o[W];
#pragma unroll
        for (int j = 0; j < W; ++j) o[j] = r * (g[i][j] - c0 - z[i][j] * c1);
        if (dskip) {
          float k[W];
          load_pack<T, W>(dskip + row * M + (long long)p * W, k);
#pragma unroll
          for (int j = 0; j < W; ++j) o[j] += k[j];
        }
        store_pack<T, W>(dxr + (long long)p * W, o);
      }
    }
  }
  if (!partial) return;
  float* out = partial + (long long)blockIdx.x * 2 * M;
  if (SUMS_IN_SMEM || blockDim.y == 1) {                 // one team in the block
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int p = i * blockDim.x + threadIdx.x;
      if (p < packs) {
#pragma unroll
        for (int j = 0; j < W; ++j) {
          out[p * W + j] = SUMS_IN_SMEM ? sums[j * packs + p] : ag[SUMS_IN_SMEM ? 0 : i][j];
          out[M + p * W + j] = SUMS_IN_SMEM ? sums[M + j * packs + p] : ab[SUMS_IN_SMEM ? 0 : i][j];
        }
      }
    }
    return;
  }
  if constexpr (!SUMS_IN_SMEM) {
    for (int t = 0; t < (int)blockDim.y; ++t) {          // the block's teams add up in order
      if ((int)threadIdx.y == t) {
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
          const int p = i * blockDim.x + threadIdx.x;
          if (p < packs) {
#pragma unroll
            for (int j = 0; j < W; ++j) {
              sums[p * W + j] = (t ? sums[p * W + j] : 0.f) + ag[i][j];
              sums[M + p * W + j] = (t ? sums[M + p * W + j] : 0.f) + ab[i][j];
            }
          }
        }
      }
      __syncthreads();
    }
    for (int c = threadIdx.y * blockDim.x + threadIdx.x; c < 2 * M; c += blockDim.x * blockDim.y) out[c] = sums[c];
  }
}

// dgamma / dbeta = sum over the partial rows, in order within each of 32 interleaved strands.
__global__ void __launch_bounds__(1024) ln_bwd_finish_kernel(const float* __restrict__ partial, int rows, int M,
                                                             float* __restrict__ dgamma, float* __restrict__ dbeta) {
  __shared__ float part[32][33];
  const int c = blockIdx.x * 32 + threadIdx.x;        // column of [dgamma | dbeta]
  float s = 0.f;
  if (c < 2 * M)
    for (int b = threadIdx.y; b < rows; b += 32) s += partial[(long long)b * 2 * M + c];
  part[threadIdx.y][threadIdx.x] = s;
  __syncthreads();
  float t = part[threadIdx.x][threadIdx.y];           // strand threadIdx.x of column threadIdx.y
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) t += __shfl_xor_sync(0xffffffffu, t, off);
  const int col = blockIdx.x * 32 + threadIdx.y;
  if (threadIdx.x == 0 && col < 2 * M) {
    if (col < M) { if (dgamma) dgamma[col] = t; }
    else if (dbeta) dbeta[col - M] = t;
  }
}

// Widest load that every row of M elements starts aligned to.
int ln_width(int M, int esize) {
  int w = 16 / esize;
  while (w > 1 && M % w) w /= 2;
  return w;
}

struct LnShape { int team, teams, nv; };   // threads per row, rows per block, values per thread

// Rows of at most 1024 elements, and many of them: one warp per row, which needs no block barrier, and 8, 16
// or 32 values per thread, eight rows per block.  Otherwise a block per row with 8 values per thread (16
// beyond 8192 elements).
LnShape ln_shape(long long n, int M) {
  LnShape s;
  if (M <= 1024 && (n >= kLnSms * 8 || M <= 256)) {
    s.nv = M <= 256 ? 8 : M <= 512 ? 16 : 32;
    s.team = 32;
    s.teams = 8;
  } else {
    s.nv = M <= 8192 ? 8 : 16;
    s.team = 32 * ceil_div(M, 32 * s.nv);
    s.teams = 1;
  }
  return s;
}

int ln_bwd_blocks(long long n, const LnShape& s) {
  const int per_sm = s.teams > 1 ? 2 : std::max(1, std::min(8, 1024 / s.team));
  const long long blocks = (n + s.teams - 1) / s.teams;
  return (int)std::min<long long>(blocks, (long long)kLnSms * per_sm);
}

template <typename T, int W>
int ln_fwd_launch(long long n, int M, float eps, const T* x, const float* gamma, const float* beta, T* y, float* mean,
                  float* rstd, cudaStream_t st) {
  const LnShape s = ln_shape(n, M);
  const dim3 block(s.team, s.teams);
  const int grid = (int)std::min<long long>((n + s.teams - 1) / s.teams, 1ll << 30);
#define GSHARD_LN(NV, NT) ln_fwd_kernel<T, W, NV / W, NT><<<grid, block, 0, st>>>(x, gamma, beta, y, mean, rstd, n, M, eps)
  if (s.teams > 1) {
    if (s.nv == 32) GSHARD_LN(32, 256);
    else if (s.nv == 16) GSHARD_LN(16, 256);
    else GSHARD_LN(8, 256);
  } else {
    if (s.nv == 16) GSHARD_LN(16, 1024);
    else GSHARD_LN(8, 1024);
  }
#undef GSHARD_LN
  count_launch();
  return cudaGetLastError() == cudaSuccess ? GSHARD_OK : GSHARD_ERR_CUDA;
}

template <typename T, int W>
int ln_bwd_launch(long long n, int M, const T* x, const float* gamma, const float* mean, const float* rstd, const T* dy,
                  const T* dskip, T* dx, float* dgamma, float* dbeta, float* partial, cudaStream_t st) {
  const LnShape s = ln_shape(n, M);
  const dim3 block(s.team, s.teams);
  const int grid = ln_bwd_blocks(n, s);
  const int smem = partial && (s.teams > 1 || s.nv == 16) ? 2 * M * (int)sizeof(float) : 0;
#define GSHARD_LN(NV, NT, SMEM)                                                                                         do {                                                                                                                    auto kern = ln_bwd_kernel<T, W, NV / W, NT, SMEM>;                                                                    if (smem > 48 * 1024 &&                                                                                                   cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) {                     cudaGetLastError();                                                                                                   return GSHARD_ERR_CUDA;                                                                                             }                                                                                                                     kern<<<grid, block, smem, st>>>(x, gamma, mean, rstd, dy, dskip, dx, partial, n, M);                                } while (0)
  if (s.teams > 1) {
    if (s.nv == 32) GSHARD_LN(32, 256, false);
    else if (s.nv == 16) GSHARD_LN(16, 256, false);
    else GSHARD_LN(8, 256, false);
  } else {
    if (s.nv == 16) GSHARD_LN(16, 1024, true);
    else GSHARD_LN(8, 1024, false);
  }
#undef GSHARD_LN
  count_launch();
  if (partial) {
    ln_bwd_finish_kernel<<<ceil_div(2 * M, 32), dim3(32, 32), 0, st>>>(partial, grid, M, dgamma, dbeta);
    count_launch();
  }
  return cudaGetLastError() == cudaSuccess ? GSHARD_OK : GSHARD_ERR_CUDA;
}

int ln_validate(int64_t n, int32_t M, int32_t dtype) {
  if (n < 0 || M <= 0) return GSHARD_ERR_INVALID_ARG;
  if (dtype != GSHARD_F32 && dtype != GSHARD_BF16) return GSHARD_ERR_INVALID_ARG;
  if (M > kLnMaxM || n > (1ll << 40) / M) return GSHARD_ERR_UNSUPPORTED_SHAPE;
  return GSHARD_OK;
}

}  // namespace

}  // namespace gshard

using namespace gshard;

extern "C" {

size_t gshard_layer_norm_workspace_bytes(int64_t n_rows, int32_t M) {
  if (ln_validate(n_rows, M, GSHARD_F32) != GSHARD_OK) return 0;
  if (n_rows == 0) return kAlign;
  return align_up((size_t)ln_bwd_blocks(n_rows, ln_shape(n_rows, M)) * 2 * M * sizeof(float));
}

int gshard_layer_norm_forward(int64_t n_rows, int32_t M, int32_t dtype, float eps, const void* x, const float* gamma,
                              const float* beta, void* y, float* mean, float* rstd, void* cuda_stream) {
  launch_counter().n = 0;
  GS_CHECK(ln_validate(n_rows, M, dtype));
  if (!(eps >= 0.f)) return GSHARD_ERR_INVALID_ARG;
  if (n_rows == 0) return GSHARD_OK;
  GS_CHECK_PTR(x); GS_CHECK_PTR(gamma); GS_CHECK_PTR(y);
  GS_CHECK_OPTIONAL_PTR(beta); GS_CHECK_OPTIONAL_PTR(mean); GS_CHECK_OPTIONAL_PTR(rstd);
  GS_CHECK(check_device());
  NvtxRange range("gshard.layer_norm");
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const int w = ln_width(M, dtype == GSHARD_BF16 ? 2 : 4);
#define GSHARD_LN_FWD(T, W) ln_fwd_launch<T, W>(n_rows, M, eps, static_cast<const T*>(x), gamma, beta, static_cast<T*>(y), mean, rstd, st)
  if (dtype == GSHARD_BF16)
    return w == 8 ? GSHARD_LN_FWD(__nv_bfloat16, 8) : w == 4 ? GSHARD_LN_FWD(__nv_bfloat16, 4)
         : w == 2 ? GSHARD_LN_FWD(__nv_bfloat16, 2) : GSHARD_LN_FWD(__nv_bfloat16, 1);
  return w == 4 ? GSHARD_LN_FWD(float, 4) : w == 2 ? GSHARD_LN_FWD(float, 2) : GSHARD_LN_FWD(float, 1);
#undef GSHARD_LN_FWD
}

int gshard_layer_norm_backward(int64_t n_rows, int32_t M, int32_t dtype, const void* x, const float* gamma,
                               const float* mean, const float* rstd, const void* dy, const void* dskip, void* dx,
                               float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  launch_counter().n = 0;
  GS_CHECK(ln_validate(n_rows, M, dtype));
  GS_CHECK_OPTIONAL_PTR(dgamma); GS_CHECK_OPTIONAL_PTR(dbeta);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (n_rows == 0) {                               // no rows: the weight gradients are empty sums
    if (!dgamma && !dbeta) return GSHARD_OK;
    GS_CHECK(check_device());
    if (dgamma && cudaMemsetAsync(dgamma, 0, (size_t)M * 4, st) != cudaSuccess) { cudaGetLastError(); return GSHARD_ERR_CUDA; }
    if (dbeta && cudaMemsetAsync(dbeta, 0, (size_t)M * 4, st) != cudaSuccess) { cudaGetLastError(); return GSHARD_ERR_CUDA; }
    return GSHARD_OK;
  }
  GS_CHECK_PTR(x); GS_CHECK_PTR(gamma); GS_CHECK_PTR(mean); GS_CHECK_PTR(rstd); GS_CHECK_PTR(dy); GS_CHECK_PTR(dx);
  GS_CHECK_OPTIONAL_PTR(dskip);
  const bool weights = dgamma || dbeta;
  if (weights) GS_CHECK_WORKSPACE(workspace, workspace_bytes, gshard_layer_norm_workspace_bytes(n_rows, M));
  GS_CHECK(check_device());
  NvtxRange range("gshard.layer_norm.backward");
  float* partial = weights ? static_cast<float*>(workspace) : nullptr;
  const int w = ln_width(M, dtype == GSHARD_BF16 ? 2 : 4);
#define GSHARD_LN_BWD(T, W)                                                                                          \
  ln_bwd_launch<T, W>(n_rows, M, static_cast<const T*>(x), gamma, mean, rstd, static_cast<const T*>(dy),             \
                      static_cast<const T*>(dskip), static_cast<T*>(dx), dgamma, dbeta, partial, st)
  if (dtype == GSHARD_BF16)
    return w == 8 ? GSHARD_LN_BWD(__nv_bfloat16, 8) : w == 4 ? GSHARD_LN_BWD(__nv_bfloat16, 4)
         : w == 2 ? GSHARD_LN_BWD(__nv_bfloat16, 2) : GSHARD_LN_BWD(__nv_bfloat16, 1);
  return w == 4 ? GSHARD_LN_BWD(float, 4) : w == 2 ? GSHARD_LN_BWD(float, 2) : GSHARD_LN_BWD(float, 1);
#undef GSHARD_LN_BWD
}

}  // extern "C"
