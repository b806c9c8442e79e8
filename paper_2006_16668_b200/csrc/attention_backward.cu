// Cross attention backward in bf16 on the tensor cores.  The scores are computed twice, once per block of keys (dk, dv)
// and once per tile of queries (dq): seven products instead of five, and every gradient is accumulated in one place
// of tensor memory in a fixed order, without atomics.
//
// Row statistics.  A first kernel writes, per tile of 128 queries, lse log2(e) and delta = sum over d of dout o in fp32, and both once
// more as three bf16 terms each, laid out as the first half of the B operand of an MMA step (the second is zeros): with ones as A
// these steps add -lse / scale to the scores and -delta to dP (24 bits, as exact as fp32), for which the threads would have to read
// shared memory that the tensor core keeps busy (32 16-byte loads per thread and tile, 900 of 3800 cycles).  The two operands share
// nothing but zeros, so that a delta that is no number stays out of P.  Rows behind the last query are padded with -1e30 for the former, so
// that their P is 0 (2^-126 at most) beside rows of dO that are zero, and nothing else needs a mask there.
//
// dk, dv: persistent CTAs; an item is 128 keys of one key head and walks the query tiles of all heads of its group.
//   S^T = K Q^T and dP^T = V dO^T into tensor memory (a thread holds 64 of a key's 128 queries), P^T over S^T, dv += P^T dO,
//   dS^T = P^T (dP^T - delta) over dP^T, dk += dS^T Q; P stays in fp32 registers between the two.  While the threads
//   work on P the tensor core runs dk of the tile before and dP^T, while they work on dS it runs dv and the next S^T; the next
//   item's first products are under way while an item's dk and dv leave tensor memory.
//   Keys behind the source's length only make rows of their own; these are written as zero.
// dq: a CTA owns 128 queries of one head and walks the source: S = Q K^T (two buffers), dP = dO V^T, dS over S,
//   dq += dS K.  Keys behind the length: dS is zero, and rows of K that hold something else are zeroed in shared memory.  dq leaves as
//   bulk tensor stores through the place of the item's last keys; stored from registers row by row, 32 lines at once, it took the
//   kernel 324 us instead of 281 at the size below.
// Both cut their walk into parts where the items do not fill the GPU.
//
// Bound by the tensor pipe and the threads' turns (a tile of dk and dv takes about 3000 cycles for 2200 of products, a block of dq 2200 for
// 1540): 16 heads of 128, 32 x 1000 x 1111 tokens, 4 key heads, kernels of 711 us: dk and dv 385, dq 281, statistics 44 (6.0 TB/s);
// 4 x 4096 x 4096 tokens 1001 us with sources of half to all of the keys.
#include <algorithm>

#include "attention.cuh"
#include "checks.cuh"
#include "pack.cuh"
#include "sm100_ptx.cuh"

namespace gshard {

namespace {

constexpr int kRows = 128;
constexpr int kThreads = 384;                 // 8 warps on the scores; TMA, MMA and two idle warps
constexpr int kScoreRegs = 216, kOtherRegs = 72;      // 2 x 128 x 216 + 128 x 72 = 384 x 168
// statistics of a query tile: lse log2(e) [128], delta [128], and the operands [128 x 8] of lse's terms and of delta's
constexpr int kTermBytes = kRows * 8 * 2, kStatFloats = 2 * kRows + 2 * kTermBytes / 4;

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// 2^x of two values without the special-function unit: x = n + f, |f| <= 1/2, 2^f by its Taylor polynomial of degree 5 (relative error
// 2.4e-6, far below the rounding of P to bf16), n into the exponent.  From 2^-126 down it stays there.
__device__ __forceinline__ float2 exp2_poly(f32x2 x2) {
  const float2 x = unpair(x2);
  float lo, hi;
  asm("max.NaN.f32 %0, %1, 0fC2FC0000;" : "=f"(lo) : "f"(x.x));
  asm("max.NaN.f32 %0, %1, 0fC2FC0000;" : "=f"(hi) : "f"(x.y));
  const f32x2 v = pair(lo, hi), t = add2(v, both(12582912.f)), f = add2(v, mul2(add2(t, both(-12582912.f)), both(-1.f)));
  f32x2 p = fma2(f, both(1.3333558e-3f), both(9.6181291e-3f));
  p = fma2(p, f, both(5.5504109e-2f));
  p = fma2(p, f, both(2.4022651e-1f));
  p = fma2(p, f, both(6.9314718e-1f));
  p = fma2(p, f, both(1.f));
  const float2 n = unpair(t);
  return unpair(mul2(p, pair(__int_as_float((__float_as_int(n.x) << 23) + 0x3f800000), __int_as_float((__float_as_int(n.y) << 23) + 0x3f800000))));
}

// 2^x of two values, pair j of a row.  The special-function unit makes 16 a cycle: with heads of up to 64 dimensions, where that takes
// as long as the products, a quarter of the pairs goes to the other unit (backward, 16 x 1024 x 1024 tokens, 16 heads of 64 on 4:
// 282 -> 267 us; with heads of 128 710 -> 720, and the forward with heads of 64 377 -> 399).
template <int DP>
__device__ __forceinline__ float2 exp2_pair(f32x2 x2, int j) {
  if (DP == 64 && j % 4 == 3) return exp2_poly(x2);
  const float2 x = unpair(x2);
  return make_float2(exp2_approx(x.x), exp2_approx(x.y));
}

// v as three bf16 terms, 16 bits of a word each from `at` on
__device__ __forceinline__ void put_terms(float v, unsigned short* out) {
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const __nv_bfloat16 t = __float2bfloat16_rn(v);
    out[i] = *reinterpret_cast<const unsigned short*>(&t);
    v -= __bfloat162float(t);
  }
}

// Exclusive prefix over the sources of the blocks of 128 keys that dk and dv have work for ([B + 1]; none without queries); one block.
__device__ void count_blocks(const AttentionArgs& a, int* prefix) {
  __shared__ int warp_sum[8];
  __shared__ int base;
  if (threadIdx.x == 0) base = 0;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int b0 = 0; b0 < a.B; b0 += 256) {
    const int b = b0 + threadIdx.x;
    const int own = b < a.B && a.Tq > 0 ? ceil_div(source_length(a, b), kRows) : 0;
    int v = own;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, v, off);
      if (lane >= off) v += o;
    }
    __syncthreads();
    if (lane == 31) warp_sum[warp] = v;
    __syncthreads();
    int before = base;
    for (int w = 0; w < warp; ++w) before += warp_sum[w];
    if (b < a.B) prefix[b] = before + v - own;
    __syncthreads();
    if (threadIdx.x == 255) base = before + v;
  }
  __syncthreads();
  if (threadIdx.x == 0) prefix[a.B] = base;
}

// A block takes 64 (query, head) rows of a tile: eight neighbouring queries of each of eight heads (so that both what lies together in o
// and dout and what lies together in the statistics is one block's), 16 lanes a row and four rows of a group in flight.  delta goes
// through shared memory, after which a thread writes all of a row.
constexpr int kStatRows = 64;
// The last block counts the sources' blocks.
__global__ void __launch_bounds__(256) attention_stats_kernel(const AttentionArgs a, float* stats, int* prefix, int q_tiles) {
  if (blockIdx.x == gridDim.x - 1) {
    count_blocks(a, prefix);
    return;
  }
  constexpr int U = kStatRows / 16;
  __shared__ float s_delta[kStatRows];
  const int part = threadIdx.x & 15, grp = threadIdx.x >> 4, c = part * 8;
  const int parts = ceil_div(kRows * a.H, kStatRows);
  const long long tile = blockIdx.x / parts;            // b * q_tiles + tile of the sequence
  const int b = (int)(tile / q_tiles), t0 = (int)(tile % q_tiles) * kRows;
  const int r0 = (int)(blockIdx.x % parts) * kStatRows;
  auto token_of = [&](int r) { return t0 + r / (8 * a.H) * 8 + r % 8; };
  auto head_of = [&](int r) { return r % (8 * a.H) / 8; };
  Pack<__nv_bfloat16, 8> x[U], y[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int r = r0 + grp + u * 16, t = token_of(r), h = head_of(r);
    x[u].raw = y[u].raw = make_uint4(0, 0, 0, 0);
    if (r < kRows * a.H && t < a.Tq && c < a.D) {
      const long long off = (((long long)b * a.Tq + t) * a.H + h) * a.D + c;
      x[u].load_once(static_cast<const __nv_bfloat16*>(a.o) + off);
      y[u].load_once(static_cast<const __nv_bfloat16*>(a.dout) + off);
    }
  }
  const int r = r0 + threadIdx.x, t = token_of(r), h = head_of(r);
  const bool mine = threadIdx.x < kStatRows && r < kRows * a.H;
  const float lse = mine && t < a.Tq ? a.lse[((long long)b * a.H + h) * a.Tq + t] : 0.f;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float delta = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) delta = fmaf(x[u].get(j), y[u].get(j), delta);
#pragma unroll
    for (int off = 8; off; off >>= 1) delta += __shfl_xor_sync(0xffffffffu, delta, off);
    if (part == 0) s_delta[grp + u * 16] = delta;
  }
  __syncthreads();
  if (!mine) return;
  const float delta = s_delta[threadIdx.x];
  float* out = stats + (((long long)b * a.H + h) * q_tiles + t0 / kRows) * kStatFloats;
  const int row = t - t0;
  out[row] = t < a.Tq ? lse * kLog2e : INFINITY;
  out[kRows + row] = delta;
  alignas(16) unsigned short terms[2][8] = {};
  put_terms(t < a.Tq ? -lse / a.scale : -1e30f, terms[0]);
  put_terms(-delta, terms[1]);
  uint4* step = reinterpret_cast<uint4*>(out + 2 * kRows) + row;
  step[0] = *reinterpret_cast<const uint4*>(terms[0]);
  step[kRows] = *reinterpret_cast<const uint4*>(terms[1]);
}

struct BackwardParams {
  AttentionArgs a;
  const float* stats;
  int q_tiles, k_tiles;
  int items;                                  // of dq
  Divisor by_tiles, by_heads, by_group;       // of q_tiles, a.H, the heads of a key head
  const int* prefix;                          // see count_blocks
  // where the items do not fill the GPU they are parts: of an item's query tiles (dk, dv), or of the source (dq)
  int kv_parts, kv_each, q_parts, q_keys;     // tiles of a part, keys of a part
  Divisor by_kv_parts, by_q_parts;
  float* part_kv; float* part_q;              // [parts][dv, dk][B, Tk, Hkv, D], [parts][B, Tq, H, D]
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

template <int DP> struct KvLayout {
  static constexpr int tile = kRows * DP * 2;
  static constexpr int stages = DP == 128 ? 2 : 4;
  static constexpr int stage = 2 * tile + 2 * kTermBytes;      // Q, dO, the terms of lse and of delta
  static constexpr int ring_off = 2 * tile;
  static constexpr int ones_off = ring_off + stages * stage;   // A operand of the terms' steps: ones in columns 0 to 2, then zeros
  static constexpr int out_off = ones_off + 2 * kTermBytes;    // 32 rows x 64 bytes per warp
  static constexpr int bar_off = out_off + 8 * 32 * 64;
  static constexpr int bytes = bar_off + 256 + 1024;
  static_assert(bytes <= 232448, "shared memory budget");
};

struct KvItem { int b, kh, k0, len, part, i0, n; };      // n query tiles to walk, from i0 on

// The i-th block of keys that has work: by source, key head, block, so that the blocks that walk the same queries run together and
// every CTA gets its share whatever the lengths are.
__device__ __forceinline__ KvItem kv_item_of(const BackwardParams& p, int i) {
  KvItem t;
  t.part = i;
  i = p.by_kv_parts.split(t.part);
  int lo = 0, hi = p.a.B - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (__ldg(p.prefix + mid) * p.a.Hkv <= i) lo = mid; else hi = mid - 1;
  }
  t.b = lo;
  const int first = __ldg(p.prefix + lo), count = __ldg(p.prefix + lo + 1) - first, r = i - first * p.a.Hkv;
  t.kh = r / count;
  t.k0 = r % count * kRows;
  t.len = source_length(p.a, lo);
  t.i0 = t.part * p.kv_each;
  t.n = min(p.kv_each, p.a.H / p.a.Hkv * p.q_tiles - t.i0);
  return t;
}
// The blocks of keys that have none are zero: the z-th of them.
__device__ __forceinline__ void zero_block(const BackwardParams& p, int z) {
  int lo = 0, hi = p.a.B - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if ((mid * p.k_tiles - __ldg(p.prefix + mid)) * p.a.Hkv <= z) lo = mid; else hi = mid - 1;
  }
  const int first = lo * p.k_tiles - __ldg(p.prefix + lo), worked = __ldg(p.prefix + lo + 1) - __ldg(p.prefix + lo);
  const int r = z - first * p.a.Hkv, kh = r / (p.k_tiles - worked), k0 = (worked + r % (p.k_tiles - worked)) * kRows;
  const int rows = min(kRows, p.a.Tk - k0);
  __nv_bfloat16* dk = static_cast<__nv_bfloat16*>(p.a.dk) + ((long long)lo * p.a.Tk + k0) * p.a.k_stride + (long long)kh * p.a.D;
  __nv_bfloat16* dv = static_cast<__nv_bfloat16*>(p.a.dv) + ((long long)lo * p.a.Tk + k0) * p.a.v_stride + (long long)kh * p.a.D;
  for (int x = threadIdx.x; x < rows * (p.a.D / 8); x += kThreads) {
    const int row = x / (p.a.D / 8), c = x % (p.a.D / 8) * 8;
    *reinterpret_cast<uint4*>(dk + row * p.a.k_stride + c) = make_uint4(0, 0, 0, 0);
    *reinterpret_cast<uint4*>(dv + row * p.a.v_stride + c) = make_uint4(0, 0, 0, 0);
  }
}

template <int DP>
__global__ void __launch_bounds__(kThreads, 1)
attention_dkv_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                     const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_do,
                     const __grid_constant__ CUtensorMap map_dk, const __grid_constant__ CUtensorMap map_dv, const BackwardParams p) {
  using L = KvLayout<DP>;
  constexpr int kStages = L::stages;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  unsigned char *sk = smem, *sv = smem + L::tile, *ring = smem + L::ring_off, *ones = smem + L::ones_off;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::bar_off);
  uint64_t* full = bars;                      // [kStages] Q, dO and their terms landed
  uint64_t* empty = full + kStages;           // [kStages]
  uint64_t* k_full = empty + kStages;
  uint64_t* k_empty = k_full + 1;
  uint64_t* v_full = k_empty + 1;
  uint64_t* v_empty = v_full + 1;
  uint64_t* s_full = v_empty + 1;
  uint64_t* dp_full = s_full + 1;
  uint64_t* p_full = dp_full + 1;             // 8 warps
  uint64_t* ds_full = p_full + 1;             // 8 warps
  uint64_t* o_full = ds_full + 1;
  uint64_t* o_empty = o_full + 1;             // 8 warps: dk and dv have left tensor memory
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(o_empty + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int group = p.a.H / p.a.Hkv;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) { ptx::mbar_init(full + s, 1); ptx::mbar_init(empty + s, 1); }
    ptx::mbar_init(k_full, 1); ptx::mbar_init(k_empty, 1); ptx::mbar_init(v_full, 1); ptx::mbar_init(v_empty, 1);
    ptx::mbar_init(s_full, 1); ptx::mbar_init(dp_full, 1);
    ptx::mbar_init(p_full, 8); ptx::mbar_init(ds_full, 8); ptx::mbar_init(o_full, 1); ptx::mbar_init(o_empty, 8);
    *abort_flag = 0;
    ptx::fence_mbar_init();
    ptx::prefetch_tensormap(&map_q);
    ptx::prefetch_tensormap(&map_do);
    ptx::prefetch_tensormap(&map_k);
    ptx::prefetch_tensormap(&map_v);
  }
  for (int x = threadIdx.x; x < 2 * kRows; x += kThreads)
    reinterpret_cast<uint4*>(ones)[x] = x < kRows ? make_uint4(0x3f803f80u, 0x3f80u, 0, 0) : make_uint4(0, 0, 0, 0);
  ptx::fence_proxy_async();
  if (warp == 9) {
    ptx::tmem_alloc(tmem_slot, 512);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  const uint32_t t_s = tmem, t_dp = tmem + 128, t_dv = tmem + 256, t_dk = tmem + 256 + DP;

  const int blocks = __ldg(p.prefix + p.a.B) * p.a.Hkv, items = blocks * p.kv_parts;
  const int zeros = p.kv_parts > 1 ? 0 : p.k_tiles * p.a.B * p.a.Hkv - blocks;      // parts: the second launch writes all of dk and dv
  for (int z = blockIdx.x; z < zeros; z += gridDim.x) zero_block(p, z);
  bool ok = true;
  if (warp >= 8) {
    ptx::registers_down<kOtherRegs>();
    if (warp == 8) {
      // ------------------------------ TMA producer -----------------------------------------------
      if (lane == 0) {
        const uint64_t again = ptx::policy_evict_last(), once = ptx::policy_evict_first();
        int stage = 0; uint32_t phase = 0, kv_phase = 0;
        for (int it = blockIdx.x; it < items && ok; it += gridDim.x) {
          const KvItem t = kv_item_of(p, it);
          if (!ptx::mbar_wait(k_empty, kv_phase ^ 1u, abort_flag)) { ok = false; break; }
          ptx::mbar_arrive_expect_tx(k_full, L::tile);
          load_rows<DP>(sk, &map_k, k_full, t.kh, t.k0, t.b, once);
          if (!ptx::mbar_wait(v_empty, kv_phase ^ 1u, abort_flag)) { ok = false; break; }
          ptx::mbar_arrive_expect_tx(v_full, L::tile);
          load_rows<DP>(sv, &map_v, v_full, t.kh, t.k0, t.b, once);
          kv_phase ^= 1u;
          for (int i = 0; i < t.n; ++i) {
            if (!ptx::mbar_wait(empty + stage, phase ^ 1u, abort_flag)) { ok = false; break; }
            int tile = t.i0 + i;
            const int h = t.kh * group + p.by_tiles.split(tile);
            unsigned char* q = ring + stage * L::stage;
            ptx::mbar_arrive_expect_tx(full + stage, L::stage);
            load_rows<DP>(q, &map_q, full + stage, h, tile * kRows, t.b, again);
            load_rows<DP>(q + L::tile, &map_do, full + stage, h, tile * kRows, t.b, again);
            ptx::bulk_load(q + 2 * L::tile, p.stats + (((long long)t.b * p.a.H + h) * p.q_tiles + tile) * kStatFloats + 2 * kRows,
                           2 * kTermBytes, full + stage);
            if (++stage == kStages) { stage = 0; phase ^= 1u; }
          }
        }
      }
    } else if (warp == 9) {
      // ------------------------------ MMA issuer (one elected thread runs all of it) ------------------
      if (ptx::elect_one()) {
        constexpr uint32_t idesc = ptx::make_idesc_bf16(kRows, kRows, false, false);
        const unsigned char* zeros = ones + kTermBytes;
        const uint32_t one = ptx::plain_desc_low(ones, zeros);
        auto wait = [&](uint64_t* bar, uint32_t parity) {
          if (ok) ok = ptx::mbar_wait(bar, parity & 1u, abort_flag);
          return ok;
        };
        int stage = 0, ahead = 0;             // of the query tile at hand, and of the tile whose scores are computed next
        uint32_t ahead_phase = 0, turn = 0, item_phase = 0, k_phase = 0, v_phase = 0;
        // scores and dP of the tile in stage `ahead`; `fresh`: the first of an item, `last`: its last
        auto scores = [&](bool fresh, bool last) {
          if (fresh) { if (!wait(k_full, k_phase)) return; k_phase ^= 1u; }
          if (!wait(full + ahead, ahead_phase)) return;
          const unsigned char* q = ring + ahead * L::stage;
          mma_rows<DP>(t_s, sk, q);
          ptx::umma_bf16_plain(t_s, one, ptx::plain_desc_low(q + 2 * L::tile, zeros), idesc, 1u);
          ptx::umma_commit(s_full);
          if (last) ptx::umma_commit(k_empty);
        };
        auto grads = [&](bool fresh, bool last) {
          if (fresh) { if (!wait(v_full, v_phase)) return; v_phase ^= 1u; }
          const unsigned char* q = ring + ahead * L::stage;
          mma_rows<DP>(t_dp, sv, q + L::tile);
          ptx::umma_bf16_plain(t_dp, one, ptx::plain_desc_low(q + 2 * L::tile + kTermBytes, zeros), idesc, 1u);
          ptx::umma_commit(dp_full);
          if (last) ptx::umma_commit(v_empty);
        };
        auto step = [&] { if (++ahead == kStages) { ahead = 0; ahead_phase ^= 1u; } };
        auto tiles_of = [&](int it) { p.by_kv_parts.split(it); return min(p.kv_each, group * p.q_tiles - it * p.kv_each); };
        int n = 0, next_n = tiles_of(blockIdx.x);
        if ((int)blockIdx.x < items) {
          scores(true, next_n == 1);
          if (ok) grads(true, next_n == 1);
          step();
        }
        for (int it = blockIdx.x; it < items && ok; it += gridDim.x) {
          const bool more = it + (int)gridDim.x < items;
          n = next_n;
          next_n = tiles_of(it + gridDim.x);
          for (int i = 0; i < n && ok; ++i) {
            const unsigned char *q = ring + stage * L::stage, *d = q + L::tile;
            const bool inner = i + 1 < n, fresh = !inner, last = inner ? i + 2 == n : next_n == 1;
            if (i == 0 && !wait(o_empty, item_phase ^ 1u)) break;       // the item before has left tensor memory
            if (!wait(p_full, turn)) break;
            ptx::tc_fence_after_sync();
            mma_weights<DP>(t_dv, t_s, d, kRows / 16, i != 0);
            if (inner || more) scores(fresh, last);
            if (!wait(ds_full, turn)) break;
            ptx::tc_fence_after_sync();
            mma_weights<DP>(t_dk, t_dp, q, kRows / 16, i != 0);
            ptx::umma_commit(empty + stage);
            if (!inner) ptx::umma_commit(o_full);
            if (inner || more) {
              grads(fresh, last);
              step();
            }
            if (++stage == kStages) stage = 0;
            turn ^= 1u;
          }
          item_phase ^= 1u;
        }
      }
    }
  } else {
    // ------------------------------ scores: two threads per key, 64 queries each -----------------------
    ptx::registers_up<kScoreRegs>();
    const int half = warp >> 2;               // queries [64 half, 64 half + 64) of a tile; later dv (0) or dk (1)
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t my_s = t_s + half * 64 + lanes, my_dp = t_dp + half * 64 + lanes;
    const f32x2 c2 = both(p.a.scale * kLog2e);
    uint32_t turn = 0, item_phase = 0;
    for (int it = blockIdx.x; it < items && ok; it += gridDim.x) {
      const KvItem t = kv_item_of(p, it);
      for (int i = 0; i < t.n; ++i) {
        if (!ptx::mbar_wait_all(s_full, turn, abort_flag)) { ok = false; break; }
        ptx::tc_fence_after_sync();
        uint32_t s[64];
        ptx::tmem_ld_32x32(my_s, s);
        ptx::tmem_ld_32x32(my_s + 32, s + 32);
        ptx::tmem_ld_wait();
        f32x2 pr[32];
        uint32_t w[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          const float2 e = exp2_pair<DP>(mul2(pair(__uint_as_float(s[2 * j]), __uint_as_float(s[2 * j + 1])), c2), j);
          pr[j] = pair(e.x, e.y);
          w[j] = pack2(e.x, e.y);
        }
        ptx::tmem_st_32x32(my_s, w);
        ptx::tmem_st_wait();
        ptx::tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(p_full);
        if (!ptx::mbar_wait_all(dp_full, turn, abort_flag)) { ok = false; break; }
        ptx::tc_fence_after_sync();
        ptx::tmem_ld_32x32(my_dp, s);
        ptx::tmem_ld_32x32(my_dp + 32, s + 32);
        ptx::tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          const float2 x = unpair(mul2(pr[j], pair(__uint_as_float(s[2 * j]), __uint_as_float(s[2 * j + 1]))));
          w[j] = pack2(x.x, x.y);
        }
        ptx::tmem_st_32x32(my_dp, w);
        ptx::tmem_st_wait();
        ptx::tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(ds_full);
        turn ^= 1u;
      }
      if (!ok || !ptx::mbar_wait_all(o_full, item_phase, abort_flag)) { ok = false; break; }
      item_phase ^= 1u;
      ptx::tc_fence_after_sync();
      // rows of dv (the first four warps) or dk through the warp's staging rows, 32 columns at a time
      const int row0 = t.k0 + (warp & 3) * 32;
      const float factor = half == 0 ? 1.f : p.a.scale;
      const bool zero = row0 + lane >= t.len;
      unsigned char* stg = smem + L::out_off + warp * 32 * 64;
      uint32_t o[DP];
#pragma unroll
      for (int j = 0; j < DP / 32; ++j) ptx::tmem_ld_32x32((half == 0 ? t_dv : t_dk) + lanes + j * 32, o + j * 32);
      ptx::tmem_ld_wait();
      ptx::tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(o_empty);
      if (p.kv_parts > 1) {                   // a part's sums, in fp32
        float* out = p.part_kv + ((((long long)(t.part * 2 + half) * p.a.B + t.b) * p.a.Tk + row0 + lane) * p.a.Hkv + t.kh) * p.a.D;
#pragma unroll
        for (int x = 0; x < DP; x += 4)
          if (!zero && x < p.a.D)
            *reinterpret_cast<float4*>(out + x) = make_float4(__uint_as_float(o[x]), __uint_as_float(o[x + 1]), __uint_as_float(o[x + 2]),
                                                              __uint_as_float(o[x + 3]));
        __syncwarp();
        continue;
      }
#pragma unroll
      for (int j = 0; j < DP / 32; ++j) {
        uint32_t w[16];
#pragma unroll
        for (int x = 0; x < 16; ++x)
          w[x] = zero ? 0u : pack2(__uint_as_float(o[j * 32 + 2 * x]) * factor, __uint_as_float(o[j * 32 + 2 * x + 1]) * factor);
        if (lane == 0) ptx::tma_store_wait_read();              // the store before has read the staging rows
        __syncwarp();
#pragma unroll
        for (int x = 0; x < 4; ++x) *reinterpret_cast<uint4*>(stg + lane * 64 + x * 16) = make_uint4(w[4 * x], w[4 * x + 1], w[4 * x + 2], w[4 * x + 3]);
        ptx::fence_proxy_async();
        __syncwarp();
        if (lane == 0 && row0 < p.a.Tk && j * 32 < p.a.D) {
          ptx::tma_store_4d(half == 0 ? &map_dv : &map_dk, stg, j * 32, t.kh, row0, t.b);
          ptx::tma_store_commit();
        }
      }
    }
    if (lane == 0) ptx::tma_store_wait_all();
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
                    const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_do,
                    const __grid_constant__ CUtensorMap map_dq, const BackwardParams p) {
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
  uint64_t* q_full = v_empty + kV;            // queries landed
  uint64_t* q_empty = q_full + 1;             // ... and have been read for the last time
  uint64_t* d_full = q_empty + 1;             // dO
  uint64_t* d_empty = d_full + 1;
  uint64_t* s_full = d_empty + 1;             // [2]
  uint64_t* dp_full = s_full + 2;
  uint64_t* ds_full = dp_full + 1;            // 8 warps: dS written, dP read
  uint64_t* o_full = ds_full + 1;
  uint64_t* k_clean = o_full + 1;             // [kK] looked through for rows behind the last key
  uint64_t* out_read = k_clean + kK;          // [kK] 8 warps: an item's dq, staged in its last keys' place, has been read
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(out_read + kK);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kK; ++s) { ptx::mbar_init(k_full + s, 1); ptx::mbar_init(k_empty + s, 2); ptx::mbar_init(k_clean + s, 1); ptx::mbar_init(out_read + s, 8); }
    for (int s = 0; s < kV; ++s) { ptx::mbar_init(v_full + s, 1); ptx::mbar_init(v_empty + s, 1); }
    ptx::mbar_init(q_full, 1); ptx::mbar_init(q_empty, 1); ptx::mbar_init(d_full, 1); ptx::mbar_init(d_empty, 1);
    ptx::mbar_init(s_full, 1); ptx::mbar_init(s_full + 1, 1); ptx::mbar_init(dp_full, 1);
    ptx::mbar_init(ds_full, 8); ptx::mbar_init(o_full, 1);
    *abort_flag = 0;
    ptx::fence_mbar_init();
    ptx::prefetch_tensormap(&map_q);
    ptx::prefetch_tensormap(&map_k);
    ptx::prefetch_tensormap(&map_v);
    ptx::prefetch_tensormap(&map_do);
    ptx::prefetch_tensormap(&map_dq);
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

  // item: part of the source (fastest), query tile, head, batch
  auto part_of = [&](int i) { p.by_q_parts.split(i); return i; };
  auto rows_of = [&](int i) { return p.by_q_parts.quotient(i); };      // the item's rows: query tile, head and batch
  auto tile_of = [&](int i) { i = rows_of(i); p.by_tiles.split(i); return i; };
  auto head_of = [&](int i) { int h = p.by_tiles.quotient(rows_of(i)); p.by_heads.split(h); return h; };
  auto batch_of = [&](int i) { return p.by_heads.quotient(p.by_tiles.quotient(rows_of(i))); };
  auto first_of = [&](int i) { return part_of(i) * p.q_keys; };        // the item's keys: the first, and how many
  auto length_of = [&](int i) { return min(max(source_length(p.a, batch_of(i)) - first_of(i), 0), p.q_keys); };
  // whether the last block has rows between its last key and the next multiple of 16, where its product ends, that TMA has not zeroed
  auto ragged = [&](int i, int len) { return (len & 15) != 0 && first_of(i) + len < p.a.Tk; };

  bool ok = true;
  if (warp >= 8) {
    ptx::registers_down<kOtherRegs>();
    if (warp == 8) {
      // ------------------------------ TMA producer -----------------------------------------------
      if (lane == 0) {
        const uint64_t again = ptx::policy_evict_last(), once = ptx::policy_evict_first();
        int ks = 0, vs = 0; uint32_t k_phase = 0, v_phase = 0, q_phase = 0;
        uint32_t staged = 0, out_phase = 0;   // bit per stage: an item's last keys are in it
        for (int i = blockIdx.x; i < p.items && ok; i += gridDim.x) {
          const int h = head_of(i), b = batch_of(i), kh = p.by_group.quotient(h), len = length_of(i), first = first_of(i);
          if (len == 0) continue;
          auto load_k = [&](int k0) {
            if (!ptx::mbar_wait(k_empty + ks, k_phase ^ 1u, abort_flag)) { ok = false; return; }
            if (staged >> ks & 1u) {
              if (!ptx::mbar_wait(out_read + ks, out_phase >> ks & 1u, abort_flag)) { ok = false; return; }
              out_phase ^= 1u << ks;
              staged ^= 1u << ks;
            }
            if (k0 + kRows >= len && p.q_parts == 1) staged |= 1u << ks;
            ptx::mbar_arrive_expect_tx(k_full + ks, L::tile);
            load_rows<DP>(sk + ks * L::tile, &map_k, k_full + ks, kh, first + k0, b, again);
            if (++ks == kK) { ks = 0; k_phase ^= 1u; }
          };
          load_k(0);
          if (!ok || !ptx::mbar_wait(q_empty, q_phase ^ 1u, abort_flag)) { ok = false; break; }
          ptx::mbar_arrive_expect_tx(q_full, L::tile);
          load_rows<DP>(sq, &map_q, q_full, h, tile_of(i) * kRows, b, once);
          if (!ptx::mbar_wait(d_empty, q_phase ^ 1u, abort_flag)) { ok = false; break; }
          ptx::mbar_arrive_expect_tx(d_full, L::tile);
          load_rows<DP>(sd, &map_do, d_full, h, tile_of(i) * kRows, b, once);
          q_phase ^= 1u;
          if (const int n = i + gridDim.x; n < p.items) {         // the next item's rows into L2: they are loaded only when these have been read
#pragma unroll
            for (int j = 0; j < DP / 64; ++j) {
              ptx::tma_prefetch_4d(&map_q, j * 64, head_of(n), tile_of(n) * kRows, batch_of(n));
              ptx::tma_prefetch_4d(&map_do, j * 64, head_of(n), tile_of(n) * kRows, batch_of(n));
            }
          }
          for (int k0 = 0; k0 < len && ok; k0 += kRows) {
            if (!ptx::mbar_wait(v_empty + vs, v_phase ^ 1u, abort_flag)) { ok = false; break; }
            ptx::mbar_arrive_expect_tx(v_full + vs, L::tile);
            load_rows<DP>(sv + vs * L::tile, &map_v, v_full + vs, kh, first + k0, b, again);
            if (++vs == kV) { vs = 0; v_phase ^= 1u; }
            if (k0 + kRows < len) load_k(k0 + kRows);
          }
        }
      }
    } else if (warp == 9) {
      // ------------------------------ MMA issuer (one elected thread runs all of it) ------------------
      if (ptx::elect_one()) {
        int ks = 0, vs = 0, ds = 0;           // ring positions of the next S, the next dP and the next dq
        uint32_t k_phase = 0, v_phase = 0, q_phase = 0, ds_phase = 0;
        auto wait = [&](uint64_t* bar, uint32_t parity) {
          if (ok) ok = ptx::mbar_wait(bar, parity, abort_flag);
          return ok;
        };
        for (int i = blockIdx.x; i < p.items && ok; i += gridDim.x) {
          const int len = length_of(i);
          if (len == 0) continue;
          const int blocks = ceil_div(len, kRows);
          auto scores = [&](int j) {
            if (!wait(k_full + ks, k_phase)) return;
            if (j == blocks - 1 && ragged(i, len) && !wait(k_clean + ks, k_phase)) return;
            mma_rows<DP>(tmem + (j & 1) * kRows, sq, sk + ks * L::tile);
            ptx::umma_commit(s_full + (j & 1));
            if (j == blocks - 1) ptx::umma_commit(q_empty);
            if (++ks == kK) { ks = 0; k_phase ^= 1u; }
          };
          auto grads = [&](int j) {           // dP of block j
            if (!wait(v_full + vs, v_phase)) return;
            mma_rows<DP>(t_dp, sd, sv + vs * L::tile);
            ptx::umma_commit(dp_full);
            ptx::umma_commit(v_empty + vs);
            if (j == blocks - 1) ptx::umma_commit(d_empty);
            if (++vs == kV) { vs = 0; v_phase ^= 1u; }
          };
          if (!wait(q_full, q_phase)) break;
          scores(0);
          if (ok && blocks > 1) scores(1);
          if (!ok || !wait(d_full, q_phase)) break;
          q_phase ^= 1u;
          grads(0);
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
        const int len = length_of(i);
        for (int k0 = 0; k0 < len; k0 += kRows) {
          if (!ptx::mbar_wait_all(k_full + ks, k_phase, abort_flag)) { ok = false; break; }
          const int left = len - k0;
          if (left <= kRows && ragged(i, len)) zero_rows<DP>(sk + ks * L::tile, left, (left + 15) & ~15, lane);
          if (lane == 0) {
            ptx::mbar_arrive(k_clean + ks);
            ptx::mbar_arrive(k_empty + ks);
          }
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
    // An item's length and its row's statistics are fetched while the item before leaves tensor memory.
    int raw = 0;
    float lse = 0.f, delta = 0.f;
    auto fetch = [&](int i) {
      if (i >= p.items) return;
      const float* stat = p.stats + (long long)rows_of(i) * kStatFloats + r;
      raw = p.a.Tk;
      if (p.a.lengths) asm volatile("ld.global.b32 %0, [%1];" : "=r"(raw) : "l"(p.a.lengths + batch_of(i)));
      asm volatile("ld.global.f32 %0, [%1];" : "=f"(lse) : "l"(stat));
      asm volatile("ld.global.f32 %0, [%1];" : "=f"(delta) : "l"(stat + kRows));
    };
    fetch(blockIdx.x);
    int stage = kK - 1;                       // of the item's last keys
    bool staged = false;                      // this warp's store may still read its place there
    for (int i = blockIdx.x; i < p.items && ok; i += gridDim.x) {
      const int h = head_of(i), b = batch_of(i), len = min(max(min(max(raw, 0), p.a.Tk) - first_of(i), 0), p.q_keys);
      const int q0 = tile_of(i) * kRows;
      const bool in = q0 + r < p.a.Tq;
      __nv_bfloat16* dq = static_cast<__nv_bfloat16*>(p.a.dq) + ((long long)b * p.a.Tq + q0 + r) * p.a.q_stride + (long long)h * p.a.D;
      if (len == 0) {
        if (in && half == 0 && p.q_parts == 1)
          for (int d = 0; d < p.a.D; d += 8) *reinterpret_cast<uint4*>(dq + d) = make_uint4(0, 0, 0, 0);
        fetch(i + gridDim.x);
        continue;
      }
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
        for (int x = 0; x < 32; ++x) {
          const float2 e = exp2_pair<DP>(fma2(pair(__uint_as_float(s[2 * x]), __uint_as_float(s[2 * x + 1])), both(c), both(-lse)), x);
          s[2 * x] = __float_as_uint(e.x);
          s[2 * x + 1] = __float_as_uint(e.y);
        }
        if (staged) {
          if (lane == 0) {
            ptx::tma_store_wait_read();
            ptx::mbar_arrive(out_read + stage);
          }
          staged = false;
        }
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
      fetch(i + gridDim.x);
      if (!ptx::mbar_wait_all(o_full, o_phase, abort_flag)) { ok = false; break; }
      o_phase ^= 1u;
      ptx::tc_fence_after_sync();
      stage = (stage + ceil_div(len, kRows)) % kK;
      if (p.q_parts > 1) {                    // a part's sums, in fp32
        float* out = p.part_q + ((((long long)part_of(i) * p.a.B + b) * p.a.Tq + q0 + r) * p.a.H + h) * p.a.D;
#pragma unroll
        for (int j = 0; j < DP / 64; ++j) {
          uint32_t o[32];
          ptx::tmem_ld_32x32(t_dq + half * (DP / 2) + j * 32 + lanes, o);
          ptx::tmem_ld_wait();
#pragma unroll
          for (int x = 0; x < 32; x += 4) {
            const int col = half * (DP / 2) + j * 32 + x;
            if (in && col < p.a.D)
              *reinterpret_cast<float4*>(out + col) = make_float4(__uint_as_float(o[x]), __uint_as_float(o[x + 1]), __uint_as_float(o[x + 2]),
                                                                  __uint_as_float(o[x + 3]));
          }
        }
      } else {
        // through the place of the item's last keys, which no product reads any more: 32 rows of DP / 2 columns per warp
        unsigned char* stg = sk + stage * L::tile + warp * 32 * DP;
        uint32_t w[DP / 4];
#pragma unroll
        for (int j = 0; j < DP / 64; ++j) {
          uint32_t o[32];
          ptx::tmem_ld_32x32(t_dq + half * (DP / 2) + j * 32 + lanes, o);
          ptx::tmem_ld_wait();
#pragma unroll
          for (int x = 0; x < 16; ++x)
            w[j * 16 + x] = pack2(__uint_as_float(o[2 * x]) * p.a.scale, __uint_as_float(o[2 * x + 1]) * p.a.scale);
        }
#pragma unroll
        for (int x = 0; x < DP / 16; ++x)     // 128-byte rows are swizzled
          *reinterpret_cast<uint4*>(stg + lane * DP + (DP == 128 ? x ^ (lane & 7) : x) * 16) = make_uint4(w[4 * x], w[4 * x + 1], w[4 * x + 2], w[4 * x + 3]);
        ptx::fence_proxy_async();
        __syncwarp();
        const int token0 = q0 + (warp & 3) * 32;
        if (lane == 0 && token0 < p.a.Tq && half * (DP / 2) < p.a.D) {
          ptx::tma_store_4d(&map_dq, stg, half * (DP / 2), h, token0, b);
          ptx::tma_store_commit();
        }
        staged = true;
      }
      ptx::tc_fence_before_sync();            // the next item's first dS says that dq has left tensor memory
    }
    if (lane == 0) ptx::tma_store_wait_all();
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
int allow_shared(K kernel, int bytes) {
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) == cudaSuccess) return GSHARD_OK;
  cudaGetLastError();
  return GSHARD_ERR_CUDA;
}

size_t prefix_floats(int B) { return ((size_t)B + 1 + 3) / 4 * 4; }        // what follows is read 16 bytes at a time
size_t rows_floats(const AttentionArgs& a) { return (size_t)a.B * a.Tq * a.H * a.D; }

// dk and dv: in query tiles of all the heads of a group; dq: in blocks of 128 keys
struct BackwardSplit { Parts kv, q; size_t kv_floats, q_floats; };
BackwardSplit split_of(const AttentionArgs& a) {
  BackwardSplit s;
  const int q_tiles = ceil_div(a.Tq, kRows), k_tiles = ceil_div(a.Tk, kRows);
  s.kv = parts_of((long long)k_tiles * a.Hkv * a.B, q_tiles * (a.H / a.Hkv), 148);
  s.q = parts_of((long long)q_tiles * a.H * a.B, k_tiles, 148);
  s.kv_floats = s.kv.parts > 1 ? (size_t)s.kv.parts * 2 * a.B * a.Tk * a.Hkv * a.D : 0;
  s.q_floats = s.q.parts > 1 ? s.q.parts * rows_floats(a) : 0;
  return s;
}

template <int DP>
int backward(const AttentionArgs& a, float* stats, cudaStream_t st) {
  BackwardParams p;
  p.a = a;
  p.stats = stats;
  p.q_tiles = ceil_div(a.Tq, kRows);
  p.k_tiles = ceil_div(a.Tk, kRows);
  const BackwardSplit split = split_of(a);
  p.kv_parts = split.kv.parts;
  p.kv_each = split.kv.each;
  p.q_parts = split.q.parts;
  p.q_keys = split.q.each * kRows;
  p.by_kv_parts = Divisor(p.kv_parts);
  p.by_q_parts = Divisor(p.q_parts);
  const int rows = p.q_tiles * a.H * a.B;     // tiles of rows
  p.items = rows * p.q_parts;
  p.by_tiles = Divisor(std::max(1, p.q_tiles));
  p.by_heads = Divisor(a.H);
  p.by_group = Divisor(a.H / a.Hkv);
  const int kv_items = p.k_tiles * a.Hkv * a.B;
  int* prefix = reinterpret_cast<int*>(stats + (size_t)rows * kStatFloats);
  p.prefix = prefix;
  p.part_kv = reinterpret_cast<float*>(prefix) + prefix_floats(a.B);
  p.part_q = p.part_kv + split.kv_floats;
  attention_stats_kernel<<<(unsigned)((long long)a.B * p.q_tiles * ceil_div(kRows * a.H, kStatRows) + 1), 256, 0, st>>>(a, stats, prefix, p.q_tiles);
  count_launch();
  CUtensorMap q, k, v, dout, dk, dv, dq;
  // Without queries or without keys the kernels write zeros and look through no map; they get valid ones all the same.
  const AttentionArgs& s = a;
  const bool both_there = a.Tq && a.Tk;
  const long long o_stride = (long long)a.H * a.D;
  const void* any = a.Tq ? a.q : a.k;
  auto map = [&](CUtensorMap* m, const void* base, int heads, int tokens, long long stride, int box_tokens, int box_dims) {
    return both_there ? make_token_map(m, base, s.D, heads, tokens, s.B, stride, box_tokens, box_dims)
                      : make_token_map(m, any, s.D, 1, 1, 1, stride, box_tokens, box_dims);
  };
  if (!map(&q, a.q, a.H, a.Tq, a.q_stride, kRows, 64) || !map(&dout, a.dout, a.H, a.Tq, o_stride, kRows, 64) ||
      !map(&k, a.k, a.Hkv, a.Tk, a.k_stride, kRows, 64) || !map(&v, a.v, a.Hkv, a.Tk, a.v_stride, kRows, 64) ||
      !map(&dk, a.dk, a.Hkv, a.Tk, a.k_stride, 32, 32) || !map(&dv, a.dv, a.Hkv, a.Tk, a.v_stride, 32, 32) ||
      !map(&dq, a.dq, a.H, a.Tq, a.q_stride, 32, DP / 2))
    return GSHARD_ERR_CUDA;
  if (kv_items) {
    GS_CHECK(allow_shared(attention_dkv_kernel<DP>, KvLayout<DP>::bytes));
    attention_dkv_kernel<DP><<<std::min(kv_items * p.kv_parts, device_sms()), kThreads, KvLayout<DP>::bytes, st>>>(q, k, v, dout, dk, dv, p);
    count_launch();
  }
  if (p.items) {
    GS_CHECK(allow_shared(attention_dq_kernel<DP>, QLayout<DP>::bytes));
    attention_dq_kernel<DP><<<std::min(p.items, device_sms()), kThreads, QLayout<DP>::bytes, st>>>(q, k, v, dout, dq, p);
    count_launch();
  }
  if (cudaGetLastError() != cudaSuccess) return GSHARD_ERR_CUDA;
  if (p.kv_parts > 1) {                       // [part][dv, dk]
    const size_t one = (size_t)a.B * a.Tk * a.Hkv * a.D;
    GS_CHECK(launch_join_gradient(a, true, p.part_kv, p.kv_parts, 0, a.dv, a.Tk, a.Hkv, a.v_stride, 1.f, st, 2 * one));
    GS_CHECK(launch_join_gradient(a, true, p.part_kv + one, p.kv_parts, 0, a.dk, a.Tk, a.Hkv, a.k_stride, a.scale, st, 2 * one));
  }
  if (p.q_parts > 1)
    GS_CHECK(launch_join_gradient(a, true, p.part_q, p.q_parts, p.q_keys, a.dq, a.Tq, a.H, a.q_stride, a.scale, st, rows_floats(a)));
  return GSHARD_OK;
}

}  // namespace

size_t attention_umma_backward_floats(const AttentionArgs& a) {
  const BackwardSplit split = split_of(a);
  return (size_t)ceil_div(a.Tq, kRows) * kStatFloats * a.H * a.B + prefix_floats(a.B) + split.kv_floats + split.q_floats;
}

int launch_attention_umma_backward(const AttentionArgs& a, float* stats, cudaStream_t st) {
  return a.D <= 64 ? backward<64>(a, stats, st) : backward<128>(a, stats, st);
}

}  // namespace gshard
