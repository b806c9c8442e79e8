// Cross attention on the CUDA cores (fp32), forward and backward: tiles of 64 queries by 64 keys, one pass over the
// keys with the running maximum and sum of the softmax, fp32 throughout.
//
// 256 threads as 16 x 16; a thread owns rows ty + 16 i and columns tx + 16 j of a score tile, or four neighbouring
// columns of an output tile.  All tiles lie in shared memory row by row with a pitch of D + 4 floats, so that the 16-byte
// reads of eight neighbouring rows fall into different banks; products take two fp32 values per instruction, along the
// head dimension for the scores and along the columns for the outputs.
// The backward takes five products per tile of scores: a block walks blocks of keys, and for each of them the queries; dk and dv stay in
// registers, dq is added to where it lies, by one block in a fixed order, without atomics.  Blocks enough for the GPU come from parts
// of the source and of the queries, with sums of their own that a second launch joins.  (8 x 517 x 333 tokens, 16 heads of 64: 417 to 452 us,
// forward 160 to 169 us; separate kernels for dq and for dk and dv, with seven products, took 550 us.)
// Bound by shared memory's operands (data pipe 78 % busy); 8 x 4 values per thread read a quarter less, but leave 8 warps per
// multiprocessor: 2 % faster with heads of 64, a fifth slower with 128.
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

// The parts of the forward's sources, `each` tiles of keys: more than one leave `out` [parts][B, Tq, H, D] and in powers of two
// `lse` [parts][B, Tq, H].
struct Split { int parts, each; float* out; float* lse; };

// acc += the same rows as stored
template <int DP>
__device__ __forceinline__ void add_tile(f32x2 (*acc)[DP / 64][2], const float* src, long long stride, int rows, int D, int tx, int ty) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < DP / 64; ++c) {
      const int r = ty + 16 * i, col = 4 * tx + 64 * c;
      if (r >= rows || col >= D) continue;
      const ulonglong2 f = *reinterpret_cast<const ulonglong2*>(src + r * stride + col);
      acc[i][c][0] = fma2(both(1.f), f.x, acc[i][c][0]);
      acc[i][c][1] = fma2(both(1.f), f.y, acc[i][c][1]);
    }
}

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

// The parts of the backward: a block walks the key blocks of one part of a source, and for each of them one part of the query tiles of
// every head that shares the keys.  More parts than one leave sums, part_q [parts of the source][B, Tq, H, D] and part_kv [parts of the
// queries][dv, dk][B, Tk, Hkv, D].
struct Cut { Parts k, q; float* part_q; float* part_kv; };

// The score tiles are computed key by query.  dk and dv stay in registers over the query tiles; dq is added to tile by tile where it
// lies, always by the same thread.
template <int DP>
__global__ void __launch_bounds__(kThreads, DP == 64 ? 2 : 1) attention_simt_backward_kernel(const AttentionArgs a, const Cut cut) {
  extern __shared__ __align__(16) float smem[];
  float *sk = smem, *sv = sk + BT * kPitch<DP>, *sq = sv + BT * kPitch<DP>, *sd = sq + BT * kPitch<DP>, *sp = sd + BT * kPitch<DP>;
  float *st = sp + BT * PP, *slse = st + BT * PP, *sdelta = slse + BT;      // st: dS query by key
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  int item = blockIdx.x;
  const int q_part = item % cut.q.parts;
  item /= cut.q.parts;
  const int k_part = item % cut.k.parts;
  item /= cut.k.parts;
  const int kh = item % a.Hkv, b = item / a.Hkv, group = a.H / a.Hkv;
  const int len = source_length(a, b), q_tiles = max(1, ceil_div(a.Tq, BT));
  const int i0 = q_part * cut.q.each, n = a.Tq ? min(i0 + cut.q.each, group * q_tiles) : i0;        // query tiles, head by head
  const int k_first = k_part * cut.k.each * BT, k_end = min(a.Tk, k_first + cut.k.each * BT), k_last = min(len, k_end);
  const float c = a.scale * kLog2e;
  auto load_do = [&](int i) {
    const int h = kh * group + i / q_tiles, q0 = i % q_tiles * BT;
    load_tile<DP>(sd, static_cast<const float*>(a.dout) + (((long long)b * a.Tq + q0) * a.H + h) * a.D, (long long)a.H * a.D,
                  i < n ? a.Tq - q0 : 0, a.D);
  };
  auto load_q = [&](int i) {
    const int h = kh * group + i / q_tiles, q0 = i % q_tiles * BT;
    load_tile<DP>(sq, static_cast<const float*>(a.q) + ((long long)b * a.Tq + q0) * a.q_stride + (long long)h * a.D, a.q_stride,
                  i < n ? a.Tq - q0 : 0, a.D);
  };
  const bool whole = cut.k.parts == 1;                  // dq itself, else the sums of a part
  const long long dq_stride = whole ? a.q_stride : (long long)a.H * a.D;
  float* const dq_base = whole ? static_cast<float*>(a.dq) : cut.part_q + (long long)k_part * a.B * a.Tq * a.H * a.D;
  auto dq_of = [&](int i) {
    return dq_base + ((long long)b * a.Tq + i % q_tiles * BT) * dq_stride + (long long)(kh * group + i / q_tiles) * a.D;
  };
  const float one[4] = {1.f, 1.f, 1.f, 1.f}, scale[4] = {a.scale, a.scale, a.scale, a.scale};
  for (int k0 = k_first; k0 < k_end; k0 += BT) {
    f32x2 dk[4][DP / 64][2], dv[4][DP / 64][2];
    clear<DP>(dk);
    clear<DP>(dv);
    const int rows = min(BT, a.Tk - k0);
    const long long koff = ((long long)b * a.Tk + k0) * a.k_stride + (long long)kh * a.D;
    const long long voff = ((long long)b * a.Tk + k0) * a.v_stride + (long long)kh * a.D;
    if (k0 < k_last) {
      __syncthreads();                                  // the last keys have been read
      load_tile<DP>(sk, static_cast<const float*>(a.k) + koff, a.k_stride, len - k0, a.D);
      load_tile<DP>(sv, static_cast<const float*>(a.v) + voff, a.v_stride, len - k0, a.D);
      load_do(i0);
      load_q(i0);
      // dO is read for the last time before Q is: its next tile is on its way during the products of dk and dq, that of Q from dq on
      for (int i = i0; i < n; ++i) {
        const int q0 = i % q_tiles * BT;
        if (threadIdx.x < BT) {
          const int t = q0 + (int)threadIdx.x;
          const long long row = ((long long)b * a.H + kh * group + i / q_tiles) * a.Tq + t;
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
            st[(tx + 16 * j) * PP + ty + 16 * x] = dp[x][j];
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
        float* const out = dq_of(i);
        f32x2 dq[4][DP / 64][2];
        clear<DP>(dq);
        if (k0 > k_first) add_tile<DP>(dq, out, dq_stride, a.Tq - q0, a.D, tx, ty);
        __syncthreads();
        load_q(i + 1);
        scores_by_rows<DP>(st, sk, dq, tx, ty);
        store_tile<DP>(out, dq_stride, a.Tq - q0, a.D, dq, whole && k0 + BT >= k_last ? scale : one, tx, ty);
      }
      landed<0>();
      // keys behind the length have gradient zero, also where dO or delta is no number and P = 0 times it is none either
#pragma unroll
      for (int x = 0; x < 4; ++x)
        if (k0 + ty + 16 * x >= len) {
#pragma unroll
          for (int d = 0; d < DP / 64; ++d) dk[x][d][0] = dk[x][d][1] = dv[x][d][0] = dv[x][d][1] = 0;
        }
    }
    if (cut.q.parts == 1) {
      store_tile<DP>(static_cast<float*>(a.dk) + koff, a.k_stride, rows, a.D, dk, scale, tx, ty);
      store_tile<DP>(static_cast<float*>(a.dv) + voff, a.v_stride, rows, a.D, dv, one, tx, ty);
    } else if (k0 < k_last) {
      const long long size = (long long)a.B * a.Tk * a.Hkv * a.D, pitch = (long long)a.Hkv * a.D;
      float* out = cut.part_kv + q_part * 2 * size + ((long long)b * a.Tk + k0) * pitch + (long long)kh * a.D;
      store_tile<DP>(out, pitch, rows, a.D, dv, one, tx, ty);
      store_tile<DP>(out + size, pitch, rows, a.D, dk, one, tx, ty);
    }
  }
  if (whole && len == 0) {
    f32x2 zero[4][DP / 64][2];
    clear<DP>(zero);
    for (int i = i0; i < n; ++i) store_tile<DP>(dq_of(i), dq_stride, a.Tq - i % q_tiles * BT, a.D, zero, one, tx, ty);
  }
}

template <typename K, typename S>
int launch(K kernel, long long blocks, int floats, const AttentionArgs& a, const S& split, cudaStream_t st) {
  const int bytes = floats * 4;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) {
    cudaGetLastError();
    return GSHARD_ERR_CUDA;
  }
  kernel<<<(unsigned)blocks, kThreads, bytes, st>>>(a, split);
  count_launch();
  return cudaGetLastError() == cudaSuccess ? GSHARD_OK : GSHARD_ERR_CUDA;
}

// shared memory holds one block per SM with heads of 128 dimensions, and registers two with 64
int slots_of(const AttentionArgs& a) { return a.D <= 64 ? 296 : 148; }
long long q_blocks(const AttentionArgs& a) { return (long long)ceil_div(a.Tq, BT) * a.H * a.B; }
Parts source_parts(const AttentionArgs& a) { return parts_of(q_blocks(a), ceil_div(a.Tk, BT), slots_of(a)); }
size_t outputs_of(const AttentionArgs& a) { return (size_t)a.B * a.Tq * a.H * a.D; }
size_t keys_of(const AttentionArgs& a) { return (size_t)a.B * a.Tk * a.Hkv * a.D; }

// The time of a cut in steps of one block of keys with one query tile (about 10 us): the work of all blocks over the slots, with a step
// for each beginning of a walk over the queries; one block's work, for the end, when slots run empty (and lengths differ); the sums of
// the parts, written and read at memory's rate.  Measured, 8 sources of at most 333 keys, 517 queries, 16 heads of 64: 682 us in one
// part, 609 in two, 423 in three, 417 in six; 8 x 512 x 2048: 3196 in one, 2746 in two, 2373 in four, 2107 in eight.
Cut cut_of(const AttentionArgs& a) {
  const int k_units = std::max(1, ceil_div(a.Tk, BT)), q_units = std::max(1, ceil_div(a.Tq, BT) * (a.H / a.Hkv));
  const long long blocks = (long long)a.B * a.Hkv, most = 8ll * slots_of(a);
  const double bytes_per_step = 50e6;
  Cut best{{1, k_units}, {1, q_units}, nullptr, nullptr};
  double least = -1;
  auto parts = [](int units, int n) { const int each = ceil_div(units, n); return Parts{ceil_div(units, each), each}; };
  for (int kn = 1; kn <= k_units && (kn == 1 || kn * blocks <= most); ++kn) {
    const Parts k = parts(k_units, kn);
    if (k.parts != kn) continue;                        // the same as fewer parts
    for (int qn = 1; qn == 1 || (qn * 4 <= q_units && qn * kn * blocks <= most); ++qn) {
      const Parts q = parts(q_units, qn);
      if (q.parts != qn) continue;
      double cost = k.each * (q.each + 1.) * (1 + (double)blocks * k.parts * q.parts / slots_of(a));
      if (k.parts > 1) cost += 1 + 8. * k.parts * outputs_of(a) / bytes_per_step;
      if (q.parts > 1) cost += 1 + 16. * q.parts * keys_of(a) / bytes_per_step;
      if (least < 0 || cost < least) { best.k = k; best.q = q; least = cost; }
    }
  }
  return best;
}
size_t part_q_floats(const AttentionArgs& a, const Cut& cut) { return cut.k.parts > 1 ? cut.k.parts * outputs_of(a) : 0; }
size_t part_kv_floats(const AttentionArgs& a, const Cut& cut) { return cut.q.parts > 1 ? cut.q.parts * 2 * keys_of(a) : 0; }

template <int DP>
int backward(const AttentionArgs& a, float* scratch, cudaStream_t st) {
  Cut cut = cut_of(a);
  cut.part_q = scratch;
  cut.part_kv = scratch + part_q_floats(a, cut);
  GS_CHECK(launch(attention_simt_backward_kernel<DP>, (long long)a.B * a.Hkv * cut.k.parts * cut.q.parts,
                  4 * BT * kPitch<DP> + 2 * BT * PP + 2 * BT, a, cut, st));
  if (cut.k.parts > 1)
    GS_CHECK(launch_join_gradient(a, false, cut.part_q, cut.k.parts, cut.k.each * BT, a.dq, a.Tq, a.H, a.q_stride, a.scale, st, outputs_of(a)));
  if (cut.q.parts > 1) {
    GS_CHECK(launch_join_gradient(a, false, cut.part_kv, cut.q.parts, 0, a.dv, a.Tk, a.Hkv, a.v_stride, 1.f, st, 2 * keys_of(a)));
    GS_CHECK(launch_join_gradient(a, false, cut.part_kv + keys_of(a), cut.q.parts, 0, a.dk, a.Tk, a.Hkv, a.k_stride, a.scale, st, 2 * keys_of(a)));
  }
  return GSHARD_OK;
}

template <int DP>
int forward(const AttentionArgs& a, float* scratch, cudaStream_t st) {
  const Parts s = source_parts(a);
  float* part_lse = scratch + (s.parts > 1 ? s.parts * outputs_of(a) : 0);
  GS_CHECK(launch(attention_simt_forward_kernel<DP>, q_blocks(a) * s.parts, 3 * BT * kPitch<DP> + BT * PP, a, Split{s.parts, s.each, scratch, part_lse},
                  st));
  return s.parts > 1 ? launch_join_outputs(a, false, scratch, part_lse, s.parts, st) : GSHARD_OK;
}

}  // namespace

size_t attention_simt_forward_floats(const AttentionArgs& a) {
  const int parts = source_parts(a).parts;
  return parts > 1 ? parts * (outputs_of(a) + (size_t)a.B * a.Tq * a.H) : 0;
}

size_t attention_simt_backward_floats(const AttentionArgs& a) {
  const Cut cut = cut_of(a);
  return part_q_floats(a, cut) + part_kv_floats(a, cut);
}

int launch_attention_simt_forward(const AttentionArgs& a, float* scratch, cudaStream_t st) {
  return a.D <= 64 ? forward<64>(a, scratch, st) : forward<128>(a, scratch, st);
}

int launch_attention_simt_backward(const AttentionArgs& a, float* scratch, cudaStream_t st) {
  return a.D <= 64 ? backward<64>(a, scratch, st) : backward<128>(a, scratch, st);
}

}  // namespace gshard
