// Cross attention on the CUDA cores (fp32), forward and backward: tiles of 64 queries by 64 keys, one pass over the
// keys with the running maximum and sum of the softmax, fp32 throughout.
//
// 256 threads as 16 x 16; a thread owns rows ty + 16 i and columns tx + 16 j of a score tile, or four neighbouring
// columns of an output tile.  All tiles lie in shared memory row by row with a pitch of D + 4 floats, so that the 16-byte
// reads of eight neighbouring rows fall into different banks; products take two fp32 values per instruction, along the
// head dimension for the scores and along the columns for the outputs.
// The backward runs over the scores twice, once per block of keys (dk, dv) and once per block of queries (dq): seven
// products instead of five, but every gradient is summed in a fixed order, without atomics.
#include "attention.cuh"
#include "checks.cuh"
#include "pack.cuh"
#include "sm100_ptx.cuh"

namespace gshard {

namespace {

constexpr int BT = 64;                  // rows of a tile
constexpr int PP = BT + 4;              // pitch of a score tile
constexpr int kThreads = 256;

template <int DP> constexpr int kPitch = DP + 4;

// 64 rows from `src` (pitch `stride` elements), asynchronously; rows from `rows` on and columns from D on are zero (nothing
// is loaded where there is no row)
template <int DP>
__device__ __forceinline__ void load_tile(float* dst, const float* src, long long stride, int rows, int D) {
  for (int i = threadIdx.x; rows > 0 && i < BT * DP / 4; i += kThreads) {
    const int r = i / (DP / 4), c = i % (DP / 4) * 4;
    const bool in = r < rows && c < D;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(ptx::smem_u32(dst + r * kPitch<DP> + c)), "l"(in ? src + r * stride + c : src),
                 "r"(in ? 16 : 0)
                 : "memory");
  }
  asm volatile("cp.async.commit_group;" ::: "memory");
}
// all but the last N tiles of this thread's have landed (for everyone behind the next barrier)
template <int N>
__device__ __forceinline__ void landed() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// s[i][j] = <row ty + 16 i of A, row tx + 16 j of B>
template <int DP>
__device__ __forceinline__ void rows_by_rows(const float* A, const float* B, float (*s)[4], int tx, int ty) {
  f32x2 acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = 0;
#pragma unroll 4
  for (int d = 0; d < DP; d += 4) {
    ulonglong2 a[4], b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = *reinterpret_cast<const ulonglong2*>(A + (ty + 16 * i) * kPitch<DP> + d);
#pragma unroll
    for (int j = 0; j < 4; ++j) b[j] = *reinterpret_cast<const ulonglong2*>(B + (tx + 16 * j) * kPitch<DP> + d);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = fma2(a[i].y, b[j].y, fma2(a[i].x, b[j].x, acc[i][j]));
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 f = unpair(acc[i][j]);
      s[i][j] = f.x + f.y;
    }
}

// acc[i][c] += sum over k of P[ty + 16 i][k] V[k][4 tx + 64 c ...]
template <int DP>
__device__ __forceinline__ void scores_by_rows(const float* P, const float* V, f32x2 (*acc)[DP / 64][2], int tx, int ty) {
#pragma unroll 2
  for (int k = 0; k < BT; k += 4) {
    float p[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 f = *reinterpret_cast<const float4*>(P + (ty + 16 * i) * PP + k);
      p[i][0] = f.x; p[i][1] = f.y; p[i][2] = f.z; p[i][3] = f.w;
    }
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
      for (int c = 0; c < DP / 64; ++c) {
        const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(V + (k + kk) * kPitch<DP> + 4 * tx + 64 * c);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          acc[i][c][0] = fma2(both(p[i][kk]), v.x, acc[i][c][0]);
          acc[i][c][1] = fma2(both(p[i][kk]), v.y, acc[i][c][1]);
        }
      }
  }
}

template <int DP>
__device__ __forceinline__ void clear(f32x2 (*acc)[DP / 64][2]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < DP / 64; ++c) acc[i][c][0] = acc[i][c][1] = 0;
}

// rows ty + 16 i below `rows` of an output tile, each times factor[i]
template <int DP>
__device__ __forceinline__ void store_tile(float* dst, long long stride, int rows, int D, f32x2 (*acc)[DP / 64][2], const float* factor, int tx,
                                           int ty) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < DP / 64; ++c) {
      const int r = ty + 16 * i, col = 4 * tx + 64 * c;
      if (r >= rows || col >= D) continue;
      const float2 lo = unpair(acc[i][c][0]), hi = unpair(acc[i][c][1]);
      const float f[4] = {lo.x * factor[i], lo.y * factor[i], hi.x * factor[i], hi.y * factor[i]};
      store_pack<float, 4>(dst + r * stride + col, f);
    }
}

// An item's part of a long axis, `each` tiles of it.  More parts than one leave their sums in `out` [parts][B, tokens, heads, D]
// (for dk and dv: dv, then dk), the forward's with their lse in powers of two, [parts][B, Tq, H].
struct Split { int parts, each; float* out; float* lse; };

template <typename F>
__device__ __forceinline__ float over_columns(float v, F f) {       // over the 16 threads of a row
#pragma unroll
  for (int off = 8; off; off >>= 1) v = f(v, __shfl_xor_sync(0xffffffffu, v, off));
  return v;
}

template <int DP>
__global__ void __launch_bounds__(kThreads) attention_simt_forward_kernel(const AttentionArgs a, const Split split) {
  extern __shared__ __align__(16) float smem[];
  float *sq = smem, *sk = sq + BT * kPitch<DP>, *sv = sk + BT * kPitch<DP>, *sp = sv + BT * kPitch<DP>;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int tiles = ceil_div(a.Tq, BT);
  const int part = blockIdx.x % split.parts, item = blockIdx.x / split.parts;
  const int q0 = item % tiles * BT, h = item / tiles % a.H, b = item / tiles / a.H;
  const int kh = h / (a.H / a.Hkv), rows = min(BT, a.Tq - q0);
  const int first = part * split.each * BT, len = min(max(source_length(a, b) - first, 0), split.each * BT);   // the part's keys
  const float* q = static_cast<const float*>(a.q) + ((long long)b * a.Tq + q0) * a.q_stride + (long long)h * a.D;
  const float* k = static_cast<const float*>(a.k) + ((long long)b * a.Tk + first) * a.k_stride + (long long)kh * a.D;
  const float* v = static_cast<const float*>(a.v) + ((long long)b * a.Tk + first) * a.v_stride + (long long)kh * a.D;
  load_tile<DP>(sq, q, a.q_stride, rows, a.D);
  f32x2 acc[4][DP / 64][2];
  clear<DP>(acc);
  float top[4], sum[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) { top[i] = -INFINITY; sum[i] = 0.f; }
  const float c = a.scale * kLog2e;
  if (len) {
    load_tile<DP>(sk, k, a.k_stride, len, a.D);
    load_tile<DP>(sv, v, a.v_stride, len, a.D);
  }
  // the next keys are on their way while the softmax and the second product run, the next values while the next scores do
  for (int k0 = 0; k0 < len; k0 += BT) {
    landed<1>();                                      // queries and keys
    __syncthreads();
    float s[4][4];
    rows_by_rows<DP>(sq, sk, s, tx, ty);
    __syncthreads();                                  // the keys have been read
    load_tile<DP>(sk, k + (k0 + BT) * a.k_stride, a.k_stride, len - k0 - BT, a.D);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float m = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (k0 + tx + 16 * j >= len) s[i][j] = -INFINITY;
        m = fmaxf(m, s[i][j]);
      }
      m = fmaxf(top[i], over_columns(m, [](float x, float y) { return fmaxf(x, y); }));
      const float ref = m == -INFINITY ? 0.f : m;
      const float shrink = exp2f((top[i] - ref) * c);
      top[i] = m;
      float t = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float p = exp2f((s[i][j] - ref) * c);
        sp[(ty + 16 * i) * PP + tx + 16 * j] = p;
        t += p;
      }
      sum[i] = fmaf(sum[i], shrink, t);
#pragma unroll
      for (int d = 0; d < DP / 64; ++d) {
        acc[i][d][0] = mul2(acc[i][d][0], both(shrink));
        acc[i][d][1] = mul2(acc[i][d][1], both(shrink));
      }
    }
    landed<1>();                                      // values
    __syncthreads();
    scores_by_rows<DP>(sp, sv, acc, tx, ty);
    __syncthreads();
    load_tile<DP>(sv, v + (k0 + BT) * a.v_stride, a.v_stride, len - k0 - BT, a.D);
  }
  landed<0>();
  float factor[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float total = over_columns(sum[i], [](float x, float y) { return x + y; });
    factor[i] = len ? 1.f / total : 0.f;
    if (tx != 0 || ty + 16 * i >= rows) continue;
    if (split.parts > 1)
      split.lse[(((long long)part * a.B + b) * a.Tq + q0 + ty + 16 * i) * a.H + h] = len ? fmaf(top[i], c, log2f(total)) : -INFINITY;
    else if (a.lse)
      a.lse[((long long)b * a.H + h) * a.Tq + q0 + ty + 16 * i] = len ? top[i] * a.scale + logf(total) : -INFINITY;
  }
  float* out = split.parts > 1 ? split.out + (long long)part * a.B * a.Tq * a.H * a.D : static_cast<float*>(a.o);
  store_tile<DP>(out + (((long long)b * a.Tq + q0) * a.H + h) * a.D, (long long)a.H * a.D, rows, a.D, acc, factor, tx, ty);
}

// dk and dv of 64 keys: the score tiles are computed key by query, over the queries of every head that shares the keys.
template <int DP>
__global__ void __launch_bounds__(kThreads) attention_simt_dkv_kernel(const AttentionArgs a, const Split split) {
  extern __shared__ __align__(16) float smem[];
  float *sk = smem, *sv = sk + BT * kPitch<DP>, *sq = sv + BT * kPitch<DP>, *sd = sq + BT * kPitch<DP>, *sp = sd + BT * kPitch<DP>;
  float *slse = sp + BT * PP, *sdelta = slse + BT;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int tiles = ceil_div(a.Tk, BT);
  const int part = blockIdx.x % split.parts, item = blockIdx.x / split.parts;
  const int k0 = item % tiles * BT, kh = item / tiles % a.Hkv, b = item / tiles / a.Hkv;
  const int len = source_length(a, b), rows = min(BT, a.Tk - k0), group = a.H / a.Hkv;
  const long long koff = ((long long)b * a.Tk + k0) * a.k_stride + (long long)kh * a.D;
  const long long voff = ((long long)b * a.Tk + k0) * a.v_stride + (long long)kh * a.D;
  f32x2 dk[4][DP / 64][2], dv[4][DP / 64][2];
  clear<DP>(dk);
  clear<DP>(dv);
  const float c = a.scale * kLog2e;
  if (k0 < len) {
    load_tile<DP>(sk, static_cast<const float*>(a.k) + koff, a.k_stride, len - k0, a.D);
    load_tile<DP>(sv, static_cast<const float*>(a.v) + voff, a.v_stride, len - k0, a.D);
    const int i0 = part * split.each, n = min(i0 + split.each, group * ceil_div(a.Tq, BT));       // query tiles, head by head
    auto head_of = [&](int i) { return kh * group + i / ceil_div(a.Tq, BT); };
    auto first_of = [&](int i) { return i % ceil_div(a.Tq, BT) * BT; };
    auto load_do = [&](int i) {
      const int h = head_of(i), q0 = first_of(i);
      load_tile<DP>(sd, static_cast<const float*>(a.dout) + (((long long)b * a.Tq + q0) * a.H + h) * a.D, (long long)a.H * a.D,
                    i < n ? a.Tq - q0 : 0, a.D);
    };
    auto load_q = [&](int i) {
      const int h = head_of(i), q0 = first_of(i);
      load_tile<DP>(sq, static_cast<const float*>(a.q) + ((long long)b * a.Tq + q0) * a.q_stride + (long long)h * a.D, a.q_stride,
                    i < n ? a.Tq - q0 : 0, a.D);
    };
    load_do(i0);
    load_q(i0);
    // dO is read for the last time before Q is: its next tile is on its way during the last product, that of Q during the first
    for (int i = i0; i < n; ++i) {
      if (threadIdx.x < BT) {
        const int t = first_of(i) + (int)threadIdx.x;
        const long long row = ((long long)b * a.H + head_of(i)) * a.Tq + t;
        const bool in = t < a.Tq;                                 // queries behind the last one: P = exp(-inf) = 0
        slse[threadIdx.x] = in ? a.lse[row] * kLog2e : INFINITY;
        sdelta[threadIdx.x] = in ? a.delta[row] : 0.f;
      }
      landed<1>();
      __syncthreads();
      float s[4][4], dp[4][4];
      rows_by_rows<DP>(sv, sd, dp, tx, ty);
      landed<0>();
      __syncthreads();
      rows_by_rows<DP>(sk, sq, s, tx, ty);
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          s[x][j] = k0 + ty + 16 * x < len ? exp2f(fmaf(s[x][j], c, -slse[tx + 16 * j])) : 0.f;
          sp[(ty + 16 * x) * PP + tx + 16 * j] = s[x][j];
          dp[x][j] = s[x][j] * (dp[x][j] - sdelta[tx + 16 * j]);
        }
      __syncthreads();
      scores_by_rows<DP>(sp, sd, dv, tx, ty);
      __syncthreads();
      load_do(i + 1);
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int j = 0; j < 4; ++j) sp[(ty + 16 * x) * PP + tx + 16 * j] = dp[x][j];
      __syncthreads();
      scores_by_rows<DP>(sp, sq, dk, tx, ty);
      __syncthreads();
      load_q(i + 1);
    }
    landed<0>();
  }
  const float one[4] = {1.f, 1.f, 1.f, 1.f}, scale[4] = {a.scale, a.scale, a.scale, a.scale};
  if (split.parts > 1) {
    if (k0 >= len) return;
    const long long size = (long long)a.B * a.Tk * a.Hkv * a.D, pitch = (long long)a.Hkv * a.D;
    float* out = split.out + part * 2 * size + ((long long)b * a.Tk + k0) * pitch + (long long)kh * a.D;
    store_tile<DP>(out, pitch, rows, a.D, dv, one, tx, ty);
    store_tile<DP>(out + size, pitch, rows, a.D, dk, one, tx, ty);
    return;
  }
  // keys behind the length have gradient zero: their scores were zero throughout
  store_tile<DP>(static_cast<float*>(a.dk) + koff, a.k_stride, rows, a.D, dk, scale, tx, ty);
  store_tile<DP>(static_cast<float*>(a.dv) + voff, a.v_stride, rows, a.D, dv, one, tx, ty);
}

template <int DP>
__global__ void __launch_bounds__(kThreads) attention_simt_dq_kernel(const AttentionArgs a, const Split split) {
  extern __shared__ __align__(16) float smem[];
  float *sq = smem, *sd = sq + BT * kPitch<DP>, *sk = sd + BT * kPitch<DP>, *sv = sk + BT * kPitch<DP>, *sp = sv + BT * kPitch<DP>;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int tiles = ceil_div(a.Tq, BT);
  const int part = blockIdx.x % split.parts, item = blockIdx.x / split.parts;
  const int q0 = item % tiles * BT, h = item / tiles % a.H, b = item / tiles / a.H;
  const int kh = h / (a.H / a.Hkv), rows = min(BT, a.Tq - q0);
  const int first = part * split.each * BT, len = min(max(source_length(a, b) - first, 0), split.each * BT);   // the part's keys
  const long long qoff = ((long long)b * a.Tq + q0) * a.q_stride + (long long)h * a.D;
  const float* k = static_cast<const float*>(a.k) + ((long long)b * a.Tk + first) * a.k_stride + (long long)kh * a.D;
  const float* v = static_cast<const float*>(a.v) + ((long long)b * a.Tk + first) * a.v_stride + (long long)kh * a.D;
  f32x2 dq[4][DP / 64][2];
  clear<DP>(dq);
  const float c = a.scale * kLog2e;
  if (len) {
    load_tile<DP>(sq, static_cast<const float*>(a.q) + qoff, a.q_stride, rows, a.D);
    load_tile<DP>(sd, static_cast<const float*>(a.dout) + (((long long)b * a.Tq + q0) * a.H + h) * a.D, (long long)a.H * a.D, rows, a.D);
    float lse[4], delta[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const long long row = ((long long)b * a.H + h) * a.Tq + q0 + ty + 16 * i;
      lse[i] = ty + 16 * i < rows ? a.lse[row] * kLog2e : INFINITY;
      delta[i] = ty + 16 * i < rows ? a.delta[row] : 0.f;
    }
    load_tile<DP>(sv, v, a.v_stride, len, a.D);
    load_tile<DP>(sk, k, a.k_stride, len, a.D);
    // the next values are on their way from the first product on, the next keys during the next first product
    for (int k0 = 0; k0 < len; k0 += BT) {
      landed<1>();
      __syncthreads();
      float s[4][4], dp[4][4];
      rows_by_rows<DP>(sd, sv, dp, tx, ty);
      landed<0>();
      __syncthreads();
      load_tile<DP>(sv, v + (k0 + BT) * a.v_stride, a.v_stride, len - k0 - BT, a.D);
      rows_by_rows<DP>(sq, sk, s, tx, ty);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          sp[(ty + 16 * i) * PP + tx + 16 * j] =
              k0 + tx + 16 * j < len ? exp2f(fmaf(s[i][j], c, -lse[i])) * (dp[i][j] - delta[i]) : 0.f;
      __syncthreads();
      scores_by_rows<DP>(sp, sk, dq, tx, ty);
      __syncthreads();
      load_tile<DP>(sk, k + (k0 + BT) * a.k_stride, a.k_stride, len - k0 - BT, a.D);
    }
    landed<0>();
  }
  if (split.parts > 1) {
    const float one[4] = {1.f, 1.f, 1.f, 1.f};
    float* out = split.out + (((long long)(part * a.B + b) * a.Tq + q0) * a.H + h) * a.D;
    if (len) store_tile<DP>(out, (long long)a.H * a.D, rows, a.D, dq, one, tx, ty);
    return;
  }
  const float scale[4] = {a.scale, a.scale, a.scale, a.scale};
  store_tile<DP>(static_cast<float*>(a.dq) + qoff, a.q_stride, rows, a.D, dq, scale, tx, ty);
}

template <typename K>
int launch(K kernel, long long blocks, int floats, const AttentionArgs& a, const Split& split, cudaStream_t st) {
  const int bytes = floats * 4;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) {
    cudaGetLastError();
    return GSHARD_ERR_CUDA;
  }
  kernel<<<(unsigned)(blocks * split.parts), kThreads, bytes, st>>>(a, split);
  count_launch();
  return cudaGetLastError() == cudaSuccess ? GSHARD_OK : GSHARD_ERR_CUDA;
}

// shared memory holds one block per SM with heads of 128 dimensions, and registers two with 64
int slots_of(const AttentionArgs& a) { return a.D <= 64 ? 296 : 148; }
long long q_blocks(const AttentionArgs& a) { return (long long)ceil_div(a.Tq, BT) * a.H * a.B; }
long long k_blocks(const AttentionArgs& a) { return (long long)ceil_div(a.Tk, BT) * a.Hkv * a.B; }
Parts source_parts(const AttentionArgs& a) { return parts_of(q_blocks(a), ceil_div(a.Tk, BT), slots_of(a)); }          // forward, dq
Parts query_parts(const AttentionArgs& a) { return parts_of(k_blocks(a), ceil_div(a.Tq, BT) * (a.H / a.Hkv), slots_of(a)); }      // dk, dv
size_t outputs_of(const AttentionArgs& a, int parts) { return parts > 1 ? (size_t)parts * a.B * a.Tq * a.H * a.D : 0; }

template <int DP>
int backward(const AttentionArgs& a, float* scratch, cudaStream_t st) {
  const int floats = 4 * BT * kPitch<DP> + BT * PP + 2 * BT;
  const Parts q = query_parts(a), s = source_parts(a);
  if (a.Tk) {
    GS_CHECK(launch(attention_simt_dkv_kernel<DP>, k_blocks(a), floats, a, Split{q.parts, q.each, scratch, nullptr}, st));
    if (q.parts > 1) {
      const size_t one = (size_t)a.B * a.Tk * a.Hkv * a.D;
      GS_CHECK(launch_join_gradient(a, false, scratch, q.parts, 0, a.dv, a.Tk, a.Hkv, a.v_stride, 1.f, st, 2 * one));
      GS_CHECK(launch_join_gradient(a, false, scratch + one, q.parts, 0, a.dk, a.Tk, a.Hkv, a.k_stride, a.scale, st, 2 * one));
    }
  }
  if (!a.Tq) return GSHARD_OK;
  GS_CHECK(launch(attention_simt_dq_kernel<DP>, q_blocks(a), floats, a, Split{s.parts, s.each, scratch, nullptr}, st));
  if (s.parts == 1) return GSHARD_OK;
  return launch_join_gradient(a, false, scratch, s.parts, s.each * BT, a.dq, a.Tq, a.H, a.q_stride, a.scale, st, outputs_of(a, s.parts) / s.parts);
}

template <int DP>
int forward(const AttentionArgs& a, float* scratch, cudaStream_t st) {
  const Parts s = source_parts(a);
  float* part_lse = scratch + outputs_of(a, s.parts);
  GS_CHECK(launch(attention_simt_forward_kernel<DP>, q_blocks(a), 3 * BT * kPitch<DP> + BT * PP, a, Split{s.parts, s.each, scratch, part_lse}, st));
  return s.parts > 1 ? launch_join_outputs(a, false, scratch, part_lse, s.parts, st) : GSHARD_OK;
}

}  // namespace

size_t attention_simt_forward_floats(const AttentionArgs& a) {
  const int parts = source_parts(a).parts;
  return parts > 1 ? outputs_of(a, parts) + (size_t)parts * a.B * a.Tq * a.H : 0;
}

// dk and dv are joined before dq's parts are written
size_t attention_simt_backward_floats(const AttentionArgs& a) {
  const int parts = query_parts(a).parts;
  return std::max(parts > 1 ? (size_t)parts * 2 * a.B * a.Tk * a.Hkv * a.D : 0, outputs_of(a, source_parts(a).parts));
}

int launch_attention_simt_forward(const AttentionArgs& a, float* scratch, cudaStream_t st) {
  return a.D <= 64 ? forward<64>(a, scratch, st) : forward<128>(a, scratch, st);
}

int launch_attention_simt_backward(const AttentionArgs& a, float* scratch, cudaStream_t st) {
  return a.D <= 64 ? backward<64>(a, scratch, st) : backward<128>(a, scratch, st);
}

}  // namespace gshard
