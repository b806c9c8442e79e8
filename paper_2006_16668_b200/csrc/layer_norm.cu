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
// Measured (bf16, 131072 x 1024): forward 93 us in a graph, 102 to 106 among single calls with new inputs (5.1 to 5.3 TB/s of
// the 6.5 a copy reaches); backward at 65536 rows with dskip 101 us, 89 of them the first kernel (6.0 TB/s).
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
// block.  `buf` holds 32 * K floats and is reused by the call after next: callers alternate two of them.
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
      for (int k = 0; k < K; ++k) buf[warp * K + k] = s[k];
    __syncthreads();
    // every thread adds the warps' sums in the same order, in two strands
    float odd[K];
#pragma unroll
    for (int k = 0; k < K; ++k) { s[k] = buf[k]; odd[k] = 0.f; }
    for (int w = 1; w < warps; w += 2) {
#pragma unroll
      for (int k = 0; k < K; ++k) {
        odd[k] += buf[w * K + k];
        if (w + 1 < warps) s[k] += buf[(w + 1) * K + k];
      }
    }
#pragma unroll
    for (int k = 0; k < K; ++k) s[k] += odd[k];
  }
}

// How the row fills the team's packs: each thread's last pack and others may be missing; none is; only last ones are.
// Knowing it saves a third of the instructions (selects and branches per element).
enum LnFill { kLnAny = 0, kLnWhole = 1, kLnLast = 2 };
#define GSHARD_LN_IN(I) (FILL == kLnWhole || (FILL == kLnLast && (I) < VPT - 1) || (I) * (int)blockDim.x + (int)threadIdx.x < packs)

// The row's values stay in registers in fp32.  AHEAD: the grid is resident, and the next row is loaded (packed)
// while the current one is worked on; in blocks of less than 1024 threads a thread also keeps its columns' gamma and
// beta in registers over all its rows (NT = 1024: 64 registers, so that two rows' blocks share a multiprocessor).
template <typename T, int W, int VPT, int NT, int MINB, bool AHEAD, int FILL>
__global__ void __launch_bounds__(NT, MINB) ln_fwd_kernel(const T* __restrict__ x, const float* __restrict__ gamma,
                                                          const float* __restrict__ beta, T* y, float* __restrict__ mean,
                                                          float* __restrict__ rstd, long long n, int M, float eps) {
  constexpr int NV = W * VPT;
  __shared__ float buf[2][32];
  constexpr bool KEEP = AHEAD && NV <= 16 && NT < 1024;
  const int packs = M / W;
  const float inv_m = 1.f / (float)M;
  const long long stride = (long long)gridDim.x * blockDim.y;
  Pack<T, W> raw[VPT];
  auto fetch = [&](long long row) {
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int p = i * blockDim.x + threadIdx.x;
      if (GSHARD_LN_IN(i)) raw[i].load_once(x + row * M + p * W);
    }
  };
  float gm[NV], bt[NV];
  auto params = [&](int i) {
    const int p = i * blockDim.x + threadIdx.x;
#pragma unroll
    for (int j = 0; j < W; ++j) gm[i * W + j] = bt[i * W + j] = 0.f;
    if (GSHARD_LN_IN(i)) {
      load_param<W>(gamma + p * W, gm + i * W);
      if (beta) load_param<W>(beta + p * W, bt + i * W);
    }
  };
  if (KEEP) {
#pragma unroll
    for (int i = 0; i < VPT; ++i) params(i);
  }
  long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y;
  if (AHEAD && row < n) fetch(row);
  for (; row < n; row += stride) {
    if (!AHEAD) fetch(row);
    float v[NV], a[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      v[j] = GSHARD_LN_IN(j / W) ? raw[j / W].get(j % W) : 0.f;
      a[j & 1] += v[j];
    }
    if (AHEAD && row + stride < n) fetch(row + stride);
    float s[1] = {a[0] + a[1]};
    team_sum<1>(s, buf[0]);
    // sum / M, rounded once: by the rounded 1 / M alone a row of 1000 x 1000 has a mean of 1000.00006, and y = -0.02
    float mu = s[0] * inv_m;
    const float left = fmaf(-mu, (float)M, s[0]);
    if (fabsf(left) < INFINITY) mu = fmaf(left, inv_m, mu);
    a[0] = a[1] = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      v[j] -= mu;
      if (!GSHARD_LN_IN(j / W)) v[j] = 0.f;     // padding stays out of the variance
      a[j & 1] = fmaf(v[j], v[j], a[j & 1]);
    }
    s[0] = a[0] + a[1];
    team_sum<1>(s, buf[1]);
    const float r = 1.f / sqrtf(s[0] * inv_m + eps);
    if (threadIdx.x == 0) {
      if (mean) mean[row] = mu;
      if (rstd) rstd[row] = r;
    }
    T* yr = y + row * M;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int p = i * blockDim.x + threadIdx.x;
      if (!KEEP) params(i);
      if (GSHARD_LN_IN(i)) {
        float o[W];
#pragma unroll
        for (int j = 0; j < W; ++j) o[j] = fmaf(v[i * W + j] * r, gm[i * W + j], bt[i * W + j]);
        store_pack<T, W>(yr + p * W, o);
      }
    }
  }
}

// Block b's share of the weight gradients goes to partial[b][0..M) (dgamma) and partial[b][M..2M) (dbeta).
// A thread's columns are summed in registers, or (SUMS_IN_SMEM, rows beyond 8192 elements, where the
// register file does not hold a row and its sums) in its own words of shared memory.  AHEAD: a team's next row
// is loaded while it works on the current one.
template <typename T, int W, int VPT, int NT, int MINB, bool AHEAD, bool SUMS_IN_SMEM, int FILL>
__global__ void __launch_bounds__(NT, MINB) ln_bwd_kernel(const T* __restrict__ x, const float* __restrict__ gamma,
                                                    const float* __restrict__ mean, const float* __restrict__ rstd, const T* dy,
                                                    const T* dskip, T* dx, float* __restrict__ partial, long long n, int M) {
  constexpr int NV = W * VPT;
  extern __shared__ float sums[];              // 2 M floats: several teams in the block, or SUMS_IN_SMEM
  __shared__ float buf[2][64];
  const int packs = M / W;
  const float inv_m = 1.f / (float)M;
  f32x2 ag[SUMS_IN_SMEM ? 1 : NV / 2], ab[SUMS_IN_SMEM ? 1 : NV / 2];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int p = j / W * blockDim.x + threadIdx.x;
    if (!SUMS_IN_SMEM) { ag[SUMS_IN_SMEM ? 0 : j / 2] = both(0.f); ab[SUMS_IN_SMEM ? 0 : j / 2] = both(0.f); }
    else if (partial && p < packs) { sums[j % W * packs + p] = 0.f; sums[M + j % W * packs + p] = 0.f; }
  }
  int flip = 0;
  const long long stride = (long long)gridDim.x * blockDim.y;
  Pack<T, W> vx[VPT], vd[VPT], vk[VPT];
  float mu = 0.f, rs = 0.f;
  auto fetch = [&](long long row, bool skip_too) {
    mu = mean[row]; rs = rstd[row];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int p = i * blockDim.x + threadIdx.x;
      const long long at = row * M + p * W;
      if (GSHARD_LN_IN(i)) {
        vx[i].load_once(x + at);
        vd[i].load_once(dy + at);
        if (skip_too) vk[i].load_once(dskip + at);
      }
    }
  };
  long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y;
  if (AHEAD && row < n) fetch(row, false);
  for (; row < n; row += stride) {
    if (!AHEAD) fetch(row, dskip != nullptr);
    f32x2 z[NV / 2], g[NV / 2];
    const float m = mu, r = rs;
#pragma unroll
    for (int j = 0; j < NV; j += 2) {
      const bool in0 = GSHARD_LN_IN(j / W);
      const bool in1 = GSHARD_LN_IN((j + 1) / W);
      const f32x2 xx = pair(in0 ? vx[j / W].get(j % W) : m, in1 ? vx[(j + 1) / W].get((j + 1) % W) : m);
      z[j / 2] = mul2(add2(xx, both(-m)), both(r));
      g[j / 2] = pair(in0 ? vd[j / W].get(j % W) : 0.f, in1 ? vd[(j + 1) / W].get((j + 1) % W) : 0.f);
    }
    if (AHEAD) {
      if (dskip) {                               // used last: loaded now, for this row
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
          const int p = i * blockDim.x + threadIdx.x;
          if (GSHARD_LN_IN(i)) vk[i].load_once(dskip + row * M + p * W);
        }
      }
      if (row + stride < n) fetch(row + stride, false);
    }
    f32x2 s0 = both(0.f), s1 = both(0.f);
    float gm[NV];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int p = i * blockDim.x + threadIdx.x;
#pragma unroll
      for (int j = 0; j < W; ++j) gm[i * W + j] = 0.f;
      if (GSHARD_LN_IN(i)) load_param<W>(gamma + p * W, gm + i * W);
    }
#pragma unroll
    for (int j = 0; j < NV; j += 2) {
      const f32x2 zz = z[j / 2], d = g[j / 2];
      if (SUMS_IN_SMEM) {
        if (partial) {
          const float2 zf = unpair(zz), df = unpair(d);
          const int p0 = j / W * blockDim.x + threadIdx.x, p1 = (j + 1) / W * blockDim.x + threadIdx.x;
          if (p0 < packs) {
            sums[j % W * packs + p0] = fmaf(df.x, zf.x, sums[j % W * packs + p0]);
            sums[M + j % W * packs + p0] += df.x;
          }
          if (p1 < packs) {
            sums[(j + 1) % W * packs + p1] = fmaf(df.y, zf.y, sums[(j + 1) % W * packs + p1]);
            sums[M + (j + 1) % W * packs + p1] += df.y;
          }
        }
      } else {
        ag[SUMS_IN_SMEM ? 0 : j / 2] = fma2(d, zz, ag[SUMS_IN_SMEM ? 0 : j / 2]);
        ab[SUMS_IN_SMEM ? 0 : j / 2] = add2(d, ab[SUMS_IN_SMEM ? 0 : j / 2]);
      }
      g[j / 2] = mul2(d, pair(gm[j], gm[j + 1]));
      s0 = add2(s0, g[j / 2]);
      s1 = fma2(g[j / 2], zz, s1);
    }
    const float2 t0 = unpair(s0), t1 = unpair(s1);
    float s[2] = {t0.x + t0.y, t1.x + t1.y};
    team_sum<2>(s, buf[flip]);
    flip ^= 1;
    const float c0 = -s[0] * inv_m, c1 = -s[1] * inv_m;
    float dxv[NV];
#pragma unroll
    for (int j = 0; j < NV; j += 2) {
      const f32x2 t = add2(fma2(z[j / 2], both(c1), g[j / 2]), both(c0));
      const f32x2 k = dskip ? pair(vk[j / W].get(j % W), vk[(j + 1) / W].get((j + 1) % W)) : both(0.f);
      const float2 o = unpair(fma2(t, both(r), k));
      dxv[j] = o.x; dxv[j + 1] = o.y;
    }
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int p = i * blockDim.x + threadIdx.x;
      if (GSHARD_LN_IN(i)) store_pack<T, W>(dx + row * M + p * W, dxv + i * W);
    }
  }
  if (!partial) return;
  float* out = partial + (long long)blockIdx.x * 2 * M;
  float fg[NV], fb[NV];                          // this thread's sums, element by element
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int p = j / W * blockDim.x + threadIdx.x;
    if (SUMS_IN_SMEM) {
      fg[j] = p < packs ? sums[j % W * packs + p] : 0.f;
      fb[j] = p < packs ? sums[M + j % W * packs + p] : 0.f;
    } else {
      const float2 u = unpair(ag[SUMS_IN_SMEM ? 0 : j / 2]), w = unpair(ab[SUMS_IN_SMEM ? 0 : j / 2]);
      fg[j] = j & 1 ? u.y : u.x;
      fb[j] = j & 1 ? w.y : w.x;
    }
  }
  if (SUMS_IN_SMEM || blockDim.y == 1) {         // one team in the block
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int p = j / W * blockDim.x + threadIdx.x;
      if (p < packs) { out[p * W + j % W] = fg[j]; out[M + p * W + j % W] = fb[j]; }
    }
    return;
  }
  if constexpr (!SUMS_IN_SMEM) {
    for (int t = 0; t < (int)blockDim.y; ++t) {          // the block's teams add up in order
      if ((int)threadIdx.y == t) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          const int p = j / W * blockDim.x + threadIdx.x;
          if (p < packs) {
            const int c = p * W + j % W;
            sums[c] = (t ? sums[c] : 0.f) + fg[j];
            sums[M + c] = (t ? sums[M + c] : 0.f) + fb[j];
          }
        }
      }
      __syncthreads();
    }
    for (int c = threadIdx.y * blockDim.x + threadIdx.x; c < 2 * M; c += blockDim.x * blockDim.y) out[c] = sums[c];
  }
}

// dgamma / dbeta = sum over the partial rows: 32 strands of rows in order, then the strands.  8 columns per
// block, so that the pass spreads over the multiprocessors.
__global__ void __launch_bounds__(256) ln_bwd_finish_kernel(const float* __restrict__ partial, int rows, int M,
                                                            float* __restrict__ dgamma, float* __restrict__ dbeta) {
  __shared__ float part[32][9];
  const int cx = threadIdx.x & 7, strand = threadIdx.x >> 3;
  const int c = blockIdx.x * 8 + cx;                  // column of [dgamma | dbeta]
  float s[4] = {0.f, 0.f, 0.f, 0.f};
  if (c < 2 * M) {
    const float* p = partial + c;
    int b = strand;
    for (; b + 96 < rows; b += 128)
#pragma unroll
      for (int k = 0; k < 4; ++k) s[k] += p[(long long)(b + 32 * k) * 2 * M];
    for (; b < rows; b += 32) s[0] += p[(long long)b * 2 * M];
  }
  part[strand][cx] = (s[0] + s[1]) + (s[2] + s[3]);
  __syncthreads();
  const int col = threadIdx.x >> 5, lane = threadIdx.x & 31;
  float t = part[lane][col];
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) t += __shfl_xor_sync(0xffffffffu, t, off);
  const int g = blockIdx.x * 8 + col;
  if (lane == 0 && g < 2 * M) {
    if (g < M) { if (dgamma) dgamma[g] = t; }
    else if (dbeta) dbeta[g - M] = t;
  }
}

// Widest load that every row of M elements starts aligned to.
int ln_width(int M, int esize) {
  int w = 16 / esize;
  while (w > 1 && M % w) w /= 2;
  return w;
}

int ln_fill(int packs, int team, int vpt) {
  return packs == team * vpt ? kLnWhole : packs >= team * (vpt - 1) ? kLnLast : kLnAny;
}

struct LnShape { int team, teams, nv; };   // threads per row, rows side by side in a block, values per thread

// Forward: one warp per row up to 1024 elements, with 8, 16 or 32 values per thread and no barrier; else a block
// per row with 16 (8 for few rows, where the latency of one row counts).
LnShape ln_fwd_shape(long long n, int M) {
  if (M <= 256) return {32, n < kLnSms * 8 ? 1 : 4, 8};
  if (n < kLnSms * 4) {
    const int nv = M <= 8192 ? 8 : 16;
    return {32 * ceil_div(M, 32 * nv), 1, nv};
  }
  if (M <= 1024) return {32, 4, M <= 512 ? 16 : 32};
  return {32 * ceil_div(M, 512), 1, 16};
}
// Backward: a thread also holds its columns' sums and its next row, so 16 values (8 of fp32, whose next row
// waits unpacked) per thread while that fits the registers.
LnShape ln_bwd_shape(int M, int esize) {
  if (M <= 256) return {32, 4, 8};
  const int nv = esize == 2 && M <= 8192 ? 16 : M <= 8192 ? 8 : 16;
  return {32 * ceil_div(M, 32 * nv), 1, nv};
}
// The backward's grid, resident as a whole: 512 threads of a multiprocessor at 128 registers each, 640 at 96.
int ln_bwd_blocks(long long n, int M, int esize) {
  const LnShape s = ln_bwd_shape(M, esize);
  const int per_sm = std::max(1, (s.nv == 16 ? 512 : 640) / (s.team * s.teams));
  return (int)std::min<long long>((n + s.teams - 1) / s.teams, (long long)kLnSms * per_sm);
}

template <typename T, int W>
int ln_fwd_launch(long long n, int M, float eps, const T* x, const float* gamma, const float* beta, T* y, float* mean,
                  float* rstd, cudaStream_t st) {
  const LnShape s = ln_fwd_shape(n, M);
  const dim3 block(s.team, s.teams);
  const long long all = (n + s.teams - 1) / s.teams;
  const int threads = s.team * s.teams;
  const bool ahead = s.nv < 32 && all > kLnSms * 4, wide = threads > 384;
  const int grid = (int)std::min<long long>(all, ahead ? kLnSms * std::max(1, (wide ? 1024 : 768) / threads) : 1ll << 30);
  const int fill = ln_fill(M / W, s.team, s.nv / W);
#define GSHARD_LN_F(NV, NT, MINB, AHEAD, FILL) \
  ln_fwd_kernel<T, W, NV / W, NT, MINB, AHEAD, FILL><<<grid, block, 0, st>>>(x, gamma, beta, y, mean, rstd, n, M, eps)
#define GSHARD_LN(NV, NT, MINB, AHEAD)                                                  \
  do {                                                                                  \
    if (W >= 4 && fill == kLnWhole) GSHARD_LN_F(NV, NT, MINB, AHEAD, (W >= 4 ? kLnWhole : kLnAny)); \
    else if (fill != kLnAny) GSHARD_LN_F(NV, NT, MINB, AHEAD, kLnLast);                 \
    else GSHARD_LN_F(NV, NT, MINB, AHEAD, kLnAny);                                      \
  } while (0)
  if (ahead && threads <= 128) { if (s.nv == 16) GSHARD_LN(16, 128, 6, true); else GSHARD_LN(8, 128, 6, true); }
  else if (ahead && !wide) GSHARD_LN(16, 384, 2, true);
  else if (ahead) GSHARD_LN(16, 1024, 1, true);
  else if (s.nv == 32) GSHARD_LN(32, 128, 8, false);
  else if (s.nv == 16) GSHARD_LN(16, 1024, 1, false);
  else GSHARD_LN(8, 1024, 1, false);
#undef GSHARD_LN
#undef GSHARD_LN_F
  count_launch();
  return cudaGetLastError() == cudaSuccess ? GSHARD_OK : GSHARD_ERR_CUDA;
}

template <typename T, int W>
int ln_bwd_launch(long long n, int M, const T* x, const float* gamma, const float* mean, const float* rstd, const T* dy,
                  const T* dskip, T* dx, float* dgamma, float* dbeta, float* partial, cudaStream_t st) {
  const LnShape s = ln_bwd_shape(M, (int)sizeof(T));
  const dim3 block(s.team, s.teams);
  const int grid = ln_bwd_blocks(n, M, (int)sizeof(T));
  const bool sums_in_smem = M > 8192;
  const int smem = partial && (s.teams > 1 || sums_in_smem) ? 2 * M * (int)sizeof(float) : 0;
  const int fill = ln_fill(M / W, s.team, s.nv / W);
  // the same limit from every call (rows have at most 16384 elements): another thread may be between its own call and launch
  constexpr int kLnBwdSmem = 2 * 16384 * (int)sizeof(float);
#define GSHARD_LN_F(NV, NT, MINB, AHEAD, SMEM, FILL)                                                                  \
  do {                                                                                                                \
    auto kern = ln_bwd_kernel<T, W, NV / W, NT, MINB, AHEAD, SMEM, FILL>;                                             \
    if (smem > 48 * 1024 &&                                                                                           \
        cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kLnBwdSmem) != cudaSuccess) {         \
      cudaGetLastError();                                                                                             \
      return GSHARD_ERR_CUDA;                                                                                         \
    }                                                                                                                 \
    kern<<<grid, block, smem, st>>>(x, gamma, mean, rstd, dy, dskip, dx, partial, n, M);                              \
  } while (0)
#define GSHARD_LN(NV, NT, MINB, AHEAD, SMEM)                                                                          \
  do {                                                                                                                \
    if (W >= 4 && fill == kLnWhole) GSHARD_LN_F(NV, NT, MINB, AHEAD, SMEM, (W >= 4 ? kLnWhole : kLnAny));             \
    else if (fill != kLnAny) GSHARD_LN_F(NV, NT, MINB, AHEAD, SMEM, kLnLast);                                         \
    else GSHARD_LN_F(NV, NT, MINB, AHEAD, SMEM, kLnAny);                                                              \
  } while (0)
  if (sums_in_smem) GSHARD_LN(16, 1024, 1, false, true);
  else if (s.nv == 16) { if constexpr (sizeof(T) == 2) GSHARD_LN(16, 512, 1, true, false); }
  else if (s.team * s.teams <= 128) GSHARD_LN(8, 128, 5, true, false);
  else if (s.team <= 640) GSHARD_LN(8, 640, 1, true, false);
  else GSHARD_LN(8, 1024, 1, false, false);
#undef GSHARD_LN
#undef GSHARD_LN_F
  count_launch();
  if (partial) {
    ln_bwd_finish_kernel<<<ceil_div(2 * M, 8), 256, 0, st>>>(partial, grid, M, dgamma, dbeta);
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
  // the type is not known here: the larger of the two grids
  const int rows = std::max(ln_bwd_blocks(n_rows, M, 2), ln_bwd_blocks(n_rows, M, 4));
  return align_up((size_t)rows * 2 * M * sizeof(float));
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
  int w = ln_width(M, dtype == GSHARD_BF16 ? 2 : 4);
  // Where gamma and beta are read again for every row (32 values per thread, or blocks too large to keep them in
  // registers), they are four times the bytes of a bf16 row: at 4 columns per lane their loads are whole 512-byte
  // passes of L1, at 8 they take twice as many (131072 x 1024: 106 against 97 us, L1 90 % busy).
  const LnShape shape = ln_fwd_shape(n_rows, M);
  if (shape.nv == 32 || shape.team > 384) w = std::min(w, 4);
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
