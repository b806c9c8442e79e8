// Cross attention backward in bf16 on the tensor cores.  The scores are computed twice, once per block of keys (dk, dv)
// and once per tile of queries (dq): seven products instead of five, and every gradient is accumulated in one place
// of tensor memory in a fixed order, without atomics and without partial sums in HBM.
//
// Row statistics.  A first kernel writes lse log2(e) and delta = sum over d of dout o per tile of 128 queries, padded with
// lse = +inf, so that P = 2^(c s - lse) of a row behind the last query is 0 and nothing else needs a mask there.
//
// dk, dv: a CTA owns 128 keys of one key head and walks the query tiles of all heads of its group.
//   S^T = K Q^T and dP^T = V dO^T into tensor memory (a thread holds 64 of a key's 128 queries), P^T over S^T, dv += P^T dO,
//   dS^T = P^T (dP^T - delta) over dP^T, dk += dS^T Q; P stays in fp32 registers between the two.  While the threads
//   work on P the tensor core runs dk of the tile before and dP^T, while they work on dS it runs dv and the next S^T.
//   Keys behind the source's length only make rows of their own; these are written as zero.
// dq: a CTA owns 128 queries of one head and walks the source: S = Q K^T (two buffers), dP = dO V^T, dS over S,
//   dq += dS K.  Keys behind the length: dS is zero, and rows of K that hold something else are zeroed in shared memory.
#include <algorithm>

#include "attention.cuh"
#include "pack.cuh"
#include "sm100_ptx.cuh"

namespace gshard {

namespace {

constexpr int kRows = 128;
constexpr int kThreads = 384;                 // 8 warps on the scores; TMA, MMA and two idle warps
constexpr int kScoreRegs = 216, kOtherRegs = 72;      // 2 x 128 x 216 + 128 x 72 = 384 x 168
constexpr int kStatBytes = 2 * kRows * 4;     // lse log2(e) and delta of a query tile

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// stats[b, h, tile][0]: lse log2(e), [1]: delta.  A block takes 64 (query, head) rows of a tile, 16 lanes a row and four rows of
// a group in flight; neighbouring rows are the heads of a token, which lie together in o and dout.
constexpr int kStatRows = 64;
__global__ void __launch_bounds__(256) attention_stats_kernel(const AttentionArgs a, float* stats, int q_tiles) {
  constexpr int U = kStatRows / 16;
  const int part = threadIdx.x & 15, grp = threadIdx.x >> 4, c = part * 8;
  const int parts = ceil_div(kRows * a.H, kStatRows);
  const long long tile = blockIdx.x / parts;            // b * q_tiles + tile of the sequence
  const int b = (int)(tile / q_tiles), t0 = (int)(tile % q_tiles) * kRows;
  const int r0 = (int)(blockIdx.x % parts) * kStatRows + grp;
  Pack<__nv_bfloat16, 8> x[U], y[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int r = r0 + u * 16, t = t0 + r / a.H, h = r % a.H;
    x[u].raw = y[u].raw = make_uint4(0, 0, 0, 0);
    if (r < kRows * a.H && t < a.Tq && c < a.D) {
      const long long off = (((long long)b * a.Tq + t) * a.H + h) * a.D + c;
      x[u].load_once(static_cast<const __nv_bfloat16*>(a.o) + off);
      y[u].load_once(static_cast<const __nv_bfloat16*>(a.dout) + off);
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int r = r0 + u * 16, t = t0 + r / a.H, h = r % a.H;
    float delta = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) delta = fmaf(x[u].get(j), y[u].get(j), delta);
#pragma unroll
    for (int off = 8; off; off >>= 1) delta += __shfl_xor_sync(0xffffffffu, delta, off);
    if (part == 0 && r < kRows * a.H) {
      const long long head = (long long)b * a.H + h;
      float* out = stats + (head * q_tiles + t0 / kRows) * (2 * kRows) + r / a.H;
      out[0] = t < a.Tq ? a.lse[head * a.Tq + t] * kLog2e : INFINITY;
      out[kRows] = delta;
    }
  }
}

struct BackwardParams {
  AttentionArgs a;
  const float* stats;
  int q_tiles, k_tiles;
  int items;                                  // dq
};

// zeroes the rows [from, to) of a tile of 128 rows x DP bf16 in two or one swizzled halves (zeros need no swizzle); whole warp
template <int DP>
__device__ __forceinline__ void zero_rows(unsigned char* tile, int from, int to, int lane) {
  for (int x = lane; x < (to - from) * (DP / 8); x += 32) {
    const int row = from + x / (DP / 8), c = x % (DP / 8);
    *reinterpret_cast<uint4*>(tile + c / 8 * (kRows * 128) + row * 128 + c % 8 * 16) = make_uint4(0, 0, 0, 0);
  }
  ptx::fence_proxy_async();
  __syncwarp();
}

template <int DP>
__device__ __forceinline__ void load_rows(unsigned char* dst, const CUtensorMap* map, uint64_t* bar, int h, int t, int b, uint64_t policy) {
#pragma unroll
  for (int j = 0; j < DP / 64; ++j) ptx::tma_load_4d(dst + j * (kRows * 128), map, bar, j * 64, h, t, b, policy);
}

// The two products, called by one elected thread.  (A branch on elect.sync, not on the lane: the compiler then knows that one
// thread issues; with lane 0 an MMA took about 170 cycles to issue instead of its 64 in the tensor core.)
// D = A B^T of two tiles in shared memory (rows by rows, along the head dimension)
template <int DP>
__device__ __forceinline__ void mma_rows(uint32_t d, const unsigned char* a, const unsigned char* b) {
  constexpr uint32_t idesc = ptx::make_idesc_bf16(kRows, kRows, false, false);
  const uint32_t da = ptx::smem_desc_low(a, 16), db = ptx::smem_desc_low(b, 16);
#pragma unroll
  for (int k = 0; k < DP / 16; ++k) {
    const uint32_t off = (uint32_t)(k / 4 * (kRows * 128) + k % 4 * 32) >> 4;
    ptx::umma_bf16_low(d, da + off, db + off, idesc, k != 0 ? 1u : 0u);
  }
}
// D (+)= A B: A is 128 x (16 steps) bf16 in tensor memory, its second 64 columns 64 tensor-memory columns behind the first;
// B a tile in shared memory whose rows are the contraction
template <int DP>
__device__ __forceinline__ void mma_weights(uint32_t d, uint32_t a, const unsigned char* b, int steps, bool add) {
  constexpr uint32_t idesc = ptx::make_idesc_bf16(kRows, DP, false, true);
  const uint32_t db = ptx::smem_desc_low(b, kRows * 128);
  auto step = [&](int k) {
    ptx::umma_bf16_ta(d, a + (k >> 2) * 64 + (k & 3) * 8, db + (uint32_t)(k * 2048 >> 4), idesc, add || k != 0 ? 1u : 0u);
  };
  if (steps == kRows / 16) {
#pragma unroll
    for (int k = 0; k < kRows / 16; ++k) step(k);
  } else {
    for (int k = 0; k < steps; ++k) step(k);
  }
}

__device__ __forceinline__ uint32_t pack2(float x, float y) {
  const __nv_bfloat162 b = __floats2bfloat162_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&b);
}

// COLS accumulator columns of this thread's row, times factor, to a row of D elements (column 0 of the thread's share is col0)
template <int COLS>
__device__ __forceinline__ void store_row(uint32_t taddr, __nv_bfloat16* out, int col0, int D, float factor, bool live, bool zero) {
#pragma unroll
  for (int j = 0; j < COLS / 32; ++j) {
    uint32_t o[32];
    ptx::tmem_ld_32x32(taddr + j * 32, o);
    ptx::tmem_ld_wait();
    if (!live) continue;
#pragma unroll
    for (int d = 0; d < 32; d += 8) {
      float f[8];
#pragma unroll
      for (int x = 0; x < 8; ++x) f[x] = zero ? 0.f : __uint_as_float(o[d + x]) * factor;
      if (col0 + j * 32 + d < D) store_pack<__nv_bfloat16, 8>(out + col0 + j * 32 + d, f);
    }
  }
}

template <int DP> struct KvLayout {
  static constexpr int tile = kRows * DP * 2;
  static constexpr int stages = 2;
  static constexpr int stage = 2 * tile;
  static constexpr int ring_off = 2 * tile;
  static constexpr int stat_off = ring_off + stages * stage;
  static constexpr int bar_off = stat_off + stages * kStatBytes;
  static constexpr int bytes = bar_off + 256 + 1024;
  static_assert(bytes <= 232448, "shared memory budget");
};

template <int DP>
__global__ void __launch_bounds__(kThreads, 1)
attention_dkv_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                     const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_do, const BackwardParams p) {
  using L = KvLayout<DP>;
  constexpr int kStages = L::stages;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  unsigned char *sk = smem, *sv = smem + L::tile, *ring = smem + L::ring_off;
  const float* stat = reinterpret_cast<const float*>(smem + L::stat_off);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::bar_off);
  uint64_t* full = bars;                      // [kStages] Q, dO and their statistics landed
  uint64_t* empty = full + kStages;           // [kStages]
  uint64_t* kv_full = empty + kStages;
  uint64_t* s_full = kv_full + 1;
  uint64_t* dp_full = s_full + 1;
  uint64_t* p_full = dp_full + 1;             // 8 warps
  uint64_t* ds_full = p_full + 1;             // 8 warps
  uint64_t* o_full = ds_full + 1;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(o_full + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  const int group = p.a.H / p.a.Hkv;
  const int k0 = blockIdx.x % p.k_tiles * kRows, kh = blockIdx.x / p.k_tiles % p.a.Hkv, b = blockIdx.x / p.k_tiles / p.a.Hkv;
  const int len = source_length(p.a, b), rows = min(kRows, p.a.Tk - k0);
  const int n = k0 < len ? group * p.q_tiles : 0;      // query tiles to walk
  __nv_bfloat16* dk = static_cast<__nv_bfloat16*>(p.a.dk) + ((long long)b * p.a.Tk + k0) * p.a.k_stride + (long long)kh * p.a.D;
  __nv_bfloat16* dv = static_cast<__nv_bfloat16*>(p.a.dv) + ((long long)b * p.a.Tk + k0) * p.a.v_stride + (long long)kh * p.a.D;
  if (n == 0) {                               // no key of this block counts, or there is no query
    for (int x = threadIdx.x; x < rows * (p.a.D / 8); x += kThreads) {
      const int r = x / (p.a.D / 8), c = x % (p.a.D / 8) * 8;
      *reinterpret_cast<uint4*>(dk + r * p.a.k_stride + c) = make_uint4(0, 0, 0, 0);
      *reinterpret_cast<uint4*>(dv + r * p.a.v_stride + c) = make_uint4(0, 0, 0, 0);
    }
    return;
  }

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) { ptx::mbar_init(full + s, 1); ptx::mbar_init(empty + s, 1); }
    ptx::mbar_init(kv_full, 1); ptx::mbar_init(s_full, 1); ptx::mbar_init(dp_full, 1);
    ptx::mbar_init(p_full, 8); ptx::mbar_init(ds_full, 8); ptx::mbar_init(o_full, 1);
    *abort_flag = 0;
    ptx::fence_mbar_init();
    ptx::prefetch_tensormap(&map_q);
    ptx::prefetch_tensormap(&map_do);
  }
  if (warp == 9) {
    ptx::tmem_alloc(tmem_slot, 512);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  const uint32_t t_s = tmem, t_dp = tmem + 128, t_dv = tmem + 256, t_dk = tmem + 256 + DP;

  bool ok = true;
  if (warp >= 8) {
    ptx::registers_down<kOtherRegs>();
    if (warp == 8) {
      // ------------------------------ TMA producer -----------------------------------------------
      if (lane == 0) {
        const uint64_t again = ptx::policy_evict_last(), once = ptx::policy_evict_first();
        ptx::mbar_arrive_expect_tx(kv_full, 2 * L::tile);
        load_rows<DP>(sk, &map_k, kv_full, kh, k0, b, once);
        load_rows<DP>(sv, &map_v, kv_full, kh, k0, b, once);
        int stage = 0; uint32_t phase = 0;
        for (int i = 0; i < n; ++i) {
          if (!ptx::mbar_wait(empty + stage, phase ^ 1u, abort_flag)) { ok = false; break; }
          const int h = kh * group + i / p.q_tiles, tile = i % p.q_tiles;
          ptx::mbar_arrive_expect_tx(full + stage, L::stage + kStatBytes);
          load_rows<DP>(ring + stage * L::stage, &map_q, full + stage, h, tile * kRows, b, again);
          load_rows<DP>(ring + stage * L::stage + L::tile, &map_do, full + stage, h, tile * kRows, b, again);
          ptx::bulk_load(smem + L::stat_off + stage * kStatBytes, p.stats + (((long long)b * p.a.H + h) * p.q_tiles + tile) * 2 * kRows,
                         kStatBytes, full + stage);
          if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
      }
    } else if (warp == 9) {
      // ------------------------------ MMA issuer (one elected thread runs all of it) ------------------
      if (ptx::elect_one()) {
        auto wait = [&](uint64_t* bar, uint32_t parity) {
          if (ok) ok = ptx::mbar_wait(bar, parity, abort_flag);
          return ok;
        };
        int stage = 0, ahead = 0;             // of query tile i, and of the tile whose scores are computed next
        uint32_t ahead_phase = 0;
        auto step = [&](int& s) { return ++s == kStages ? (s = 0, true) : false; };
        if (wait(kv_full, 0) && wait(full, 0)) {
          mma_rows<DP>(t_s, sk, ring);
          ptx::umma_commit(s_full);
          mma_rows<DP>(t_dp, sv, ring + L::tile);
          ptx::umma_commit(dp_full);
        }
        if (step(ahead)) ahead_phase ^= 1u;
        for (int i = 0; i < n && ok; ++i) {
          const unsigned char *q = ring + stage * L::stage, *d = q + L::tile;
          const unsigned char *q1 = ring + ahead * L::stage, *d1 = q1 + L::tile;
          const bool more = i + 1 < n;
          if (more && !wait(full + ahead, ahead_phase)) break;
          if (!wait(p_full, i & 1)) break;
          ptx::tc_fence_after_sync();
          mma_weights<DP>(t_dv, t_s, d, kRows / 16, i != 0);
          if (more) {
            mma_rows<DP>(t_s, sk, q1);
            ptx::umma_commit(s_full);
          }
          if (!wait(ds_full, i & 1)) break;
          ptx::tc_fence_after_sync();
          mma_weights<DP>(t_dk, t_dp, q, kRows / 16, i != 0);
          ptx::umma_commit(empty + stage);
          if (more) {
            mma_rows<DP>(t_dp, sv, d1);
            ptx::umma_commit(dp_full);
          } else {
            ptx::umma_commit(o_full);
          }
          step(stage);
          if (step(ahead)) ahead_phase ^= 1u;
        }
      }
    }
  } else {
    // ------------------------------ scores: a thread per key, two threads' worth of queries -----------
    ptx::registers_up<kScoreRegs>();
    const int half = warp >> 2;               // queries [64 half, 64 half + 64) of a tile
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t my_s = t_s + half * 64 + lanes, my_dp = t_dp + half * 64 + lanes;
    const float c = p.a.scale * kLog2e;
    int stage = 0; uint32_t phase = 0;
    for (int i = 0; i < n; ++i) {
      const float4* lse4 = reinterpret_cast<const float4*>(stat + stage * 2 * kRows + half * 64);
      const float4* delta4 = lse4 + kRows / 4;
      bool here = ptx::mbar_wait(full + stage, phase, abort_flag) && ptx::mbar_wait(s_full, i & 1, abort_flag);
      if (!__all_sync(0xffffffffu, here)) { ok = false; break; }
      ptx::tc_fence_after_sync();
      uint32_t s[64];
      ptx::tmem_ld_32x32(my_s, s);
      ptx::tmem_ld_32x32(my_s + 32, s + 32);
      ptx::tmem_ld_wait();
      uint32_t w[32];
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const float4 l = lse4[j];
        const float m[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
        for (int x = 0; x < 4; ++x) s[4 * j + x] = __float_as_uint(exp2_approx(fmaf(__uint_as_float(s[4 * j + x]), c, -m[x])));
        w[2 * j] = pack2(__uint_as_float(s[4 * j]), __uint_as_float(s[4 * j + 1]));
        w[2 * j + 1] = pack2(__uint_as_float(s[4 * j + 2]), __uint_as_float(s[4 * j + 3]));
      }
      ptx::tmem_st_32x32(my_s, w);
      ptx::tmem_st_wait();
      ptx::tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(p_full);
      here = ptx::mbar_wait(dp_full, i & 1, abort_flag);
      if (!__all_sync(0xffffffffu, here)) { ok = false; break; }
      ptx::tc_fence_after_sync();
      uint32_t g[64];
      ptx::tmem_ld_32x32(my_dp, g);
      ptx::tmem_ld_32x32(my_dp + 32, g + 32);
      ptx::tmem_ld_wait();
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const float4 l = delta4[j];
        const float m[4] = {l.x, l.y, l.z, l.w};
        float f[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) f[x] = __uint_as_float(s[4 * j + x]) * (__uint_as_float(g[4 * j + x]) - m[x]);
        w[2 * j] = pack2(f[0], f[1]);
        w[2 * j + 1] = pack2(f[2], f[3]);
      }
      ptx::tmem_st_32x32(my_dp, w);
      ptx::tmem_st_wait();
      ptx::tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(ds_full);
      if (++stage == kStages) { stage = 0; phase ^= 1u; }
    }
    if (ok && !__all_sync(0xffffffffu, ptx::mbar_wait(o_full, 0, abort_flag))) ok = false;
    if (ok) {
      ptx::tc_fence_after_sync();
      const int r = threadIdx.x & 127;
      const bool zero = k0 + r >= len;
      if (half == 0) store_row<DP>(t_dv + lanes, dv + r * p.a.v_stride, 0, p.a.D, 1.f, r < rows, zero);
      else store_row<DP>(t_dk + lanes, dk + r * p.a.k_stride, 0, p.a.D, p.a.scale, r < rows, zero);
    }
  }

  if (!ok) {
    *abort_flag = 1;
    set_device_status(p.a.status, GSHARD_ERR_TIMEOUT);
    const uint64_t t0 = ptx::globaltimer_ns();
    while (ptx::globaltimer_ns() - t0 < 2000000ull) { __nanosleep(1000); }
  }
  __syncwarp();
  ptx::tc_fence_before_sync();
  __syncthreads();
  if (warp == 9) {
    ptx::tc_fence_after_sync();
    ptx::tmem_dealloc(tmem, 512);
  }
}

template <int DP> struct QLayout {
  static constexpr int tile = kRows * DP * 2;
  static constexpr int k_stages = 3, v_stages = 2;
  static constexpr int k_off = 2 * tile;
  static constexpr int v_off = k_off + k_stages * tile;
  static constexpr int bar_off = v_off + v_stages * tile;
  static constexpr int bytes = std::max(bar_off + 256 + 1024, 120 * 1024);      // one CTA per multiprocessor: all of tensor memory
  static_assert(bytes <= 232448, "shared memory budget");
};

template <int DP>
__global__ void __launch_bounds__(kThreads, 1)
attention_dq_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                    const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_do, const BackwardParams p) {
  using L = QLayout<DP>;
  constexpr int kK = L::k_stages, kV = L::v_stages;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  unsigned char *sq = smem, *sd = smem + L::tile, *sk = smem + L::k_off, *sv = smem + L::v_off;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::bar_off);
  uint64_t* k_full = bars;
  uint64_t* k_empty = k_full + kK;            // MMA, cleaning warp
  uint64_t* v_full = k_empty + kK;
  uint64_t* v_empty = v_full + kV;
  uint64_t* q_full = v_empty + kV;            // queries and dO landed
  uint64_t* q_empty = q_full + 1;
  uint64_t* s_full = q_empty + 1;             // [2]
  uint64_t* dp_full = s_full + 2;
  uint64_t* ds_full = dp_full + 1;            // 8 warps: dS written, dP read
  uint64_t* o_full = ds_full + 1;
  uint64_t* k_clean = o_full + 1;             // rows behind the last key zeroed
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(k_clean + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int group = p.a.H / p.a.Hkv;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kK; ++s) { ptx::mbar_init(k_full + s, 1); ptx::mbar_init(k_empty + s, 2); }
    ptx::mbar_init(k_clean, 1);
    for (int s = 0; s < kV; ++s) { ptx::mbar_init(v_full + s, 1); ptx::mbar_init(v_empty + s, 1); }
    ptx::mbar_init(q_full, 1); ptx::mbar_init(q_empty, 1);
    ptx::mbar_init(s_full, 1); ptx::mbar_init(s_full + 1, 1); ptx::mbar_init(dp_full, 1);
    ptx::mbar_init(ds_full, 8); ptx::mbar_init(o_full, 1);
    *abort_flag = 0;
    ptx::fence_mbar_init();
    ptx::prefetch_tensormap(&map_q);
    ptx::prefetch_tensormap(&map_k);
    ptx::prefetch_tensormap(&map_v);
    ptx::prefetch_tensormap(&map_do);
  }
  if (warp == 9) {
    ptx::tmem_alloc(tmem_slot, 512);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;           // S (two buffers), dP, dq
  const uint32_t t_dp = tmem + 256, t_dq = tmem + 384;

  // item: query tile (fastest), head, batch
  auto head_of = [&](int i) { return i / p.q_tiles % p.a.H; };
  auto batch_of = [&](int i) { return i / p.q_tiles / p.a.H; };
  // whether the last block has rows between its last key and the next multiple of 16, where its product ends, that TMA has not zeroed
  auto ragged = [&](int len) { return (len & 15) != 0 && len < p.a.Tk; };

  bool ok = true;
  if (warp >= 8) {
    ptx::registers_down<kOtherRegs>();
    if (warp == 8) {
      // ------------------------------ TMA producer -----------------------------------------------
      if (lane == 0) {
        const uint64_t again = ptx::policy_evict_last(), once = ptx::policy_evict_first();
        int ks = 0, vs = 0; uint32_t k_phase = 0, v_phase = 0, q_phase = 0;
        for (int i = blockIdx.x; i < p.items && ok; i += gridDim.x) {
          const int h = head_of(i), b = batch_of(i), kh = h / group, len = source_length(p.a, b);
          if (len == 0) continue;
          auto load_k = [&](int k0) {
            if (!ptx::mbar_wait(k_empty + ks, k_phase ^ 1u, abort_flag)) { ok = false; return; }
            ptx::mbar_arrive_expect_tx(k_full + ks, L::tile);
            load_rows<DP>(sk + ks * L::tile, &map_k, k_full + ks, kh, k0, b, again);
            if (++ks == kK) { ks = 0; k_phase ^= 1u; }
          };
          load_k(0);
          if (!ok || !ptx::mbar_wait(q_empty, q_phase ^ 1u, abort_flag)) { ok = false; break; }
          q_phase ^= 1u;
          ptx::mbar_arrive_expect_tx(q_full, 2 * L::tile);
          load_rows<DP>(sq, &map_q, q_full, h, i % p.q_tiles * kRows, b, once);
          load_rows<DP>(sd, &map_do, q_full, h, i % p.q_tiles * kRows, b, once);
          for (int k0 = 0; k0 < len && ok; k0 += kRows) {
            if (!ptx::mbar_wait(v_empty + vs, v_phase ^ 1u, abort_flag)) { ok = false; break; }
            ptx::mbar_arrive_expect_tx(v_full + vs, L::tile);
            load_rows<DP>(sv + vs * L::tile, &map_v, v_full + vs, kh, k0, b, again);
            if (++vs == kV) { vs = 0; v_phase ^= 1u; }
            if (k0 + kRows < len) load_k(k0 + kRows);
          }
        }
      }
    } else if (warp == 9) {
      // ------------------------------ MMA issuer (one elected thread runs all of it) ------------------
      if (ptx::elect_one()) {
        int ks = 0, vs = 0, ds = 0;           // ring positions of the next S, the next dP and the next dq
        uint32_t k_phase = 0, v_phase = 0, q_phase = 0, ds_phase = 0, clean_phase = 0;
        auto wait = [&](uint64_t* bar, uint32_t parity) {
          if (ok) ok = ptx::mbar_wait(bar, parity, abort_flag);
          return ok;
        };
        for (int i = blockIdx.x; i < p.items && ok; i += gridDim.x) {
          const int len = source_length(p.a, batch_of(i));
          if (len == 0) continue;
          const int blocks = ceil_div(len, kRows);
          auto scores = [&](int j) {
            if (!wait(k_full + ks, k_phase)) return;
            if (j == blocks - 1 && ragged(len)) {
              if (!wait(k_clean, clean_phase)) return;
              clean_phase ^= 1u;
            }
            mma_rows<DP>(tmem + (j & 1) * kRows, sq, sk + ks * L::tile);
            ptx::umma_commit(s_full + (j & 1));
            if (++ks == kK) { ks = 0; k_phase ^= 1u; }
          };
          auto grads = [&](int j) {           // dP of block j
            if (!wait(v_full + vs, v_phase)) return;
            mma_rows<DP>(t_dp, sd, sv + vs * L::tile);
            ptx::umma_commit(dp_full);
            ptx::umma_commit(v_empty + vs);
            if (j == blocks - 1) ptx::umma_commit(q_empty);
            if (++vs == kV) { vs = 0; v_phase ^= 1u; }
          };
          if (!wait(q_full, q_phase)) break;
          q_phase ^= 1u;
          scores(0);
          // a block's scores always go before its dP, so that "queries read" may follow the last dP
          if (ok && blocks > 1) scores(1);
          if (ok) grads(0);
          for (int j = 0; j < blocks && ok; ++j) {
            if (!wait(ds_full, ds_phase)) break;
            ptx::tc_fence_after_sync();
            ds_phase ^= 1u;
            const int steps = min(kRows, (len - j * kRows + 15) & ~15) / 16;
            if (j + 1 < blocks) grads(j + 1);   // first: the threads are about to wait for it
            if (!ok) break;
            mma_weights<DP>(t_dq, tmem + (j & 1) * kRows, sk + ds * L::tile, steps, j != 0);
            ptx::umma_commit(k_empty + ds);
            if (j == blocks - 1) ptx::umma_commit(o_full);
            if (++ds == kK) ds = 0;
            if (j + 2 < blocks) scores(j + 2);
          }
        }
      }
    } else if (warp == 10) {
      // ------------------------------ zeroes what lies behind a source's last key ----------------------
      // It follows every stage, so that no phase of the barriers passes by unseen.
      int ks = 0; uint32_t k_phase = 0;
      for (int i = blockIdx.x; i < p.items && ok; i += gridDim.x) {
        const int len = source_length(p.a, batch_of(i));
        for (int k0 = 0; k0 < len; k0 += kRows) {
          if (!ptx::mbar_wait_all(k_full + ks, k_phase, abort_flag)) { ok = false; break; }
          const int left = len - k0;
          if (left <= kRows && ragged(len)) {
            zero_rows<DP>(sk + ks * L::tile, left, (left + 15) & ~15, lane);
            if (lane == 0) ptx::mbar_arrive(k_clean);
          }
          if (lane == 0) ptx::mbar_arrive(k_empty + ks);
          if (++ks == kK) { ks = 0; k_phase ^= 1u; }
        }
      }
    }
  } else {
    // ------------------------------ scores: two threads per query, 64 keys each ------------------------
    ptx::registers_up<kScoreRegs>();
    const int half = warp >> 2;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const float c = p.a.scale * kLog2e;
    const int r = threadIdx.x & 127;
    uint32_t s_phase[2] = {0, 0}, dp_phase = 0, o_phase = 0;
    for (int i = blockIdx.x; i < p.items && ok; i += gridDim.x) {
      const int h = head_of(i), b = batch_of(i), len = source_length(p.a, b);
      const int q0 = i % p.q_tiles * kRows;
      const bool in = q0 + r < p.a.Tq;
      __nv_bfloat16* dq = static_cast<__nv_bfloat16*>(p.a.dq) + ((long long)b * p.a.Tq + q0 + r) * p.a.q_stride + (long long)h * p.a.D;
      if (len == 0) {
        if (in && half == 0)
          for (int d = 0; d < p.a.D; d += 8) *reinterpret_cast<uint4*>(dq + d) = make_uint4(0, 0, 0, 0);
        continue;
      }
      const float* stat = p.stats + (long long)i * 2 * kRows;
      const float lse = __ldg(stat + r), delta = __ldg(stat + kRows + r);
      for (int j = 0; j * kRows < len; ++j) {
        const uint32_t my_s = tmem + (j & 1) * kRows + half * 64 + lanes, my_dp = t_dp + half * 64 + lanes;
        bool here = ptx::mbar_wait(s_full + (j & 1), s_phase[j & 1], abort_flag);
        s_phase[j & 1] ^= 1u;
        if (!__all_sync(0xffffffffu, here)) { ok = false; break; }
        ptx::tc_fence_after_sync();
        uint32_t s[64], g[64];
        ptx::tmem_ld_32x32(my_s, s);
        ptx::tmem_ld_32x32(my_s + 32, s + 32);
        ptx::tmem_ld_wait();
#pragma unroll
        for (int x = 0; x < 64; ++x) s[x] = __float_as_uint(exp2_approx(fmaf(__uint_as_float(s[x]), c, -lse)));
        here = ptx::mbar_wait(dp_full, dp_phase, abort_flag);
        dp_phase ^= 1u;
        if (!__all_sync(0xffffffffu, here)) { ok = false; break; }
        ptx::tc_fence_after_sync();
        ptx::tmem_ld_32x32(my_dp, g);
        ptx::tmem_ld_32x32(my_dp + 32, g + 32);
        ptx::tmem_ld_wait();
        float f[64];
#pragma unroll
        for (int x = 0; x < 64; ++x) f[x] = __uint_as_float(s[x]) * (__uint_as_float(g[x]) - delta);
        const int left = len - j * kRows - half * 64;
        if (left < 64) {
#pragma unroll
          for (int x = 0; x < 64; ++x)
            if (x >= left) f[x] = 0.f;
        }
        uint32_t w[32];
#pragma unroll
        for (int x = 0; x < 32; ++x) w[x] = pack2(f[2 * x], f[2 * x + 1]);
        ptx::tmem_st_32x32(my_s, w);
        ptx::tmem_st_wait();
        ptx::tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(ds_full);
      }
      if (!ok) break;
      if (!ptx::mbar_wait_all(o_full, o_phase, abort_flag)) { ok = false; break; }
      o_phase ^= 1u;
      ptx::tc_fence_after_sync();
      store_row<DP / 2>(t_dq + half * (DP / 2) + lanes, dq, half * (DP / 2), p.a.D, p.a.scale, in, false);
      ptx::tc_fence_before_sync();            // the next item's first dS says that dq has left tensor memory
    }
  }

  if (!ok) {
    *abort_flag = 1;
    set_device_status(p.a.status, GSHARD_ERR_TIMEOUT);
    const uint64_t t0 = ptx::globaltimer_ns();
    while (ptx::globaltimer_ns() - t0 < 2000000ull) { __nanosleep(1000); }
  }
  __syncwarp();
  ptx::tc_fence_before_sync();
  __syncthreads();
  if (warp == 9) {
    ptx::tc_fence_after_sync();
    ptx::tmem_dealloc(tmem, 512);
  }
}

template <typename K>
int launch(K kernel, int blocks, int bytes, const CUtensorMap* m, const BackwardParams& p, cudaStream_t st) {
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) {
    cudaGetLastError();
    return GSHARD_ERR_CUDA;
  }
  kernel<<<blocks, kThreads, bytes, st>>>(m[0], m[1], m[2], m[3], p);
  count_launch();
  return cudaGetLastError() == cudaSuccess ? GSHARD_OK : GSHARD_ERR_CUDA;
}

template <int DP>
int backward(const AttentionArgs& a, float* stats, cudaStream_t st) {
  BackwardParams p;
  p.a = a;
  p.stats = stats;
  p.q_tiles = ceil_div(a.Tq, kRows);
  p.k_tiles = ceil_div(a.Tk, kRows);
  p.items = p.q_tiles * a.H * a.B;
  if (p.items) {
    attention_stats_kernel<<<(unsigned)((long long)a.B * p.q_tiles * ceil_div(kRows * a.H, kStatRows)), 256, 0, st>>>(a, stats, p.q_tiles);
    count_launch();
  }
  CUtensorMap m[4] = {};
  // without queries no kernel looks at a map
  if (a.Tq && (!make_token_map(&m[0], a.q, a.D, a.H, a.Tq, a.B, a.q_stride, kRows) || !make_source_map(&m[1], a, a.k, a.k_stride, kRows) ||
               !make_source_map(&m[2], a, a.v, a.v_stride, kRows) ||
               !make_token_map(&m[3], a.dout, a.D, a.H, a.Tq, a.B, (long long)a.H * a.D, kRows)))
    return GSHARD_ERR_CUDA;
  if (a.Tk) {
    const int rc = launch(attention_dkv_kernel<DP>, p.k_tiles * a.Hkv * a.B, KvLayout<DP>::bytes, m, p, st);
    if (rc != GSHARD_OK) return rc;
  }
  if (!a.Tq) return GSHARD_OK;
  return launch(attention_dq_kernel<DP>, std::min(p.items, device_sms()), QLayout<DP>::bytes, m, p, st);
}

}  // namespace

size_t attention_stats_floats(int B, int Tq, int H) { return (size_t)ceil_div(Tq, kRows) * 2 * kRows * H * B; }

int launch_attention_umma_backward(const AttentionArgs& a, float* stats, cudaStream_t st) {
  return a.D <= 64 ? backward<64>(a, stats, st) : backward<128>(a, stats, st);
}

}  // namespace gshard
