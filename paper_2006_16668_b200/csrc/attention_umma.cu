// Cross attention forward in bf16 on the tensor cores (tcgen05, accumulators in tensor memory), one pass over the keys.
//
// A CTA owns two tiles of 128 query rows that share a key head and walks the source in blocks of 128 keys.  Per block and tile:
// S = Q K^T into 128 columns of tensor memory; one thread per row reads its scores, takes the block's maximum, writes
// p = 2^(c (s - m)) as bf16 over the scores, and the second product O += P V reads P from tensor memory.  While the four warps of one tile work on their scores, the
// tensor core runs the other tile's products.  The issue order S0 | S1, then PV0, S0', PV1, S1' ... makes every hand-over of a
// buffer a consequence of the in-order execution of MMAs:
//   scores of block j+1 overwrite P of block j behind the PV product that read it;
//   "scores complete" of block j+1 also says that PV of block j is complete, so that O may be rescaled.
// O is rescaled only when a row's maximum has grown by more than 2^8 since the last time (the weights then stay below
// 2^8, and their sums far from overflow); that is rare after the first blocks.
// Persistent grid, one CTA per multiprocessor, and the stream of products does not stop between two items: the scores of the
// next item follow the last block's, and a fourth warpgroup takes the finished output from tensor memory, divides it by its sums
// and sends it off through shared memory (bulk tensor stores) while the next item's first block is being worked on.
//
// Where the items do not fill the GPU and the source is long, an item is one of several parts of the source: it leaves its output in fp32
// and the logarithm of its sums, and a second launch joins them in order (one head, 64 queries, 32768 keys: 46 us).
//
// Rows behind the source's length: scores are masked before the maximum; rows of V that hold something else are zeroed in
// shared memory up to the next multiple of 16, where the last block's product ends.
//
// Bound by the turns between exponentials and products: heads of 128, 16 of them, 4 x 4096 x 4096 tokens 437 us (1.26 PFLOP/s), 64 x 1024 x
// 1024 481 us (1.14); sources of 512 to 1024 keys 424 to 454 us, since a block that has one key takes as long as a full
// one (768 keys 377 us, 769 439).  Leaving out the exponentials behind a last block's keys made the kernel larger and all sizes 4 %
// slower; blocks of 64 keys were slower as well.
#include <algorithm>

#include "attention.cuh"
#include "pack.cuh"
#include "sm100_ptx.cuh"

namespace gshard {

namespace {

constexpr int kRows = 128;                    // query rows of a tile, keys of a block
constexpr int kThreads = 512;                 // 2 x 4 softmax warps; 4 output warps; TMA, MMA and two idle warps
// registers per thread: 128 at launch, moved to where the scores live (128 x (2 x 184 + 80 + 64) = 512 x 128)
constexpr int kSoftmaxRegs = 184, kOutputRegs = 80, kOtherRegs = 64;
constexpr float kSlack = 8.f;                 // growth of a row's maximum (powers of two) that O is not rescaled for

template <int DP> struct Layout {
  static constexpr int tile = kRows * DP * 2;
  static constexpr int stage = 2 * tile;                       // values of a block, and the keys that come after it
  static constexpr int stages = DP == 128 ? 2 : 3;
  static constexpr int kv_off = 2 * tile;
  static constexpr int out_off = kv_off + stages * stage;      // 32 rows x 128 bytes per output warp
  static constexpr int stat_off = out_off + 4 * 32 * 128;      // sum and maximum of every row of both tiles
  static constexpr int bar_off = stat_off + 2 * 2 * kRows * 4;
  static constexpr int bytes = bar_off + 256 + 1024;
  static_assert(bytes <= 232448, "shared memory budget");
};

struct Tile { int h, q0, rows; };             // rows: (token from q0 on, one of the tile's heads from h on), heads fastest

struct Item {
  int b, kh, first, tiles;                    // the tiles first, first + 1 (or only the first) of the key head's list
  int part, k0, len;                          // keys [k0, k0 + len)
};

struct ForwardParams {
  AttentionArgs a;
  int group;                                  // heads of a key head
  int heads, tokens;                          // of a tile: all heads of a group where they are 1, 2, 4, .. 32, else one; 128 / heads
  int q_tiles;                                // tiles of a sequence
  int list;                                   // tiles per key head
  int pairs;                                  // items per key head and part
  int items;
  Divisor by_parts, by_pairs, by_kv_heads, by_tiles, by_heads;      // of parts, pairs, a.Hkv, q_tiles, heads
  int parts, part_keys;                       // parts of a source, a multiple of 128 keys each
  float* part_o; float* part_lse;             // parts > 1: [parts][B, Tq, H, D] and (powers of two) [parts][B, Tq, H]
};

__device__ __forceinline__ Item item_of(const ForwardParams& p, int i) {
  Item t;
  t.part = i;                                  // fastest, then the pair of tiles, the key head, the source
  t.first = p.by_parts.split(t.part);
  t.kh = p.by_pairs.split(t.first);
  t.b = p.by_kv_heads.split(t.kh);
  t.first *= 2;
  t.tiles = min(2, p.list - t.first);
  t.k0 = t.part * p.part_keys;
  t.len = min(max(source_length(p.a, t.b) - t.k0, 0), p.part_keys);
  return t;
}
__device__ __forceinline__ Tile tile_of(const ForwardParams& p, const Item& t, int half) {
  int i = t.first + half;
  const int heads = p.by_tiles.split(i);
  Tile r;
  r.h = t.kh * p.group + heads * p.heads;
  r.q0 = i * p.tokens;
  r.rows = min(p.tokens, p.a.Tq - r.q0) * p.heads;
  return r;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

template <int DP>
__global__ void __launch_bounds__(kThreads, 1)
attention_umma_forward_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                              const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_o, const ForwardParams p) {
  using L = Layout<DP>;
  constexpr int kStages = L::stages;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  unsigned char* ring = smem + L::kv_off;
  float* stat = reinterpret_cast<float*>(smem + L::stat_off);     // [tile][sum, maximum][row]
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::bar_off);
  uint64_t* kv_full = bars;                   // [kStages]
  uint64_t* kv_empty = kv_full + kStages;     // [kStages] (MMA, cleaning warp)
  uint64_t* q_full = kv_empty + kStages;      // [2] a tile's queries landed
  uint64_t* q_empty = q_full + 2;             // [2] ... and have been read for the last time
  uint64_t* s_full = q_empty + 2;             // [2] scores complete
  uint64_t* p_full = s_full + 2;              // [2] weights written (4 warps)
  uint64_t* o_full = p_full + 2;              // [2] output complete
  uint64_t* o_empty = o_full + 2;             // [2] output and statistics read (4 warps)
  uint64_t* stat_full = o_empty + 2;          // [2] statistics written (4 warps)
  uint64_t* v_clean = stat_full + 2;          // [kStages] looked through for rows behind the last key
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(v_clean + kStages);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) { ptx::mbar_init(kv_full + s, 1); ptx::mbar_init(kv_empty + s, 2); ptx::mbar_init(v_clean + s, 1); }
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(q_full + i, 1); ptx::mbar_init(q_empty + i, 1);
      ptx::mbar_init(s_full + i, 1); ptx::mbar_init(p_full + i, 4);
      ptx::mbar_init(o_full + i, 1); ptx::mbar_init(o_empty + i, 4); ptx::mbar_init(stat_full + i, 4);
    }
    *abort_flag = 0;
    ptx::fence_mbar_init();
    ptx::prefetch_tensormap(&map_q);
    ptx::prefetch_tensormap(&map_k);
    ptx::prefetch_tensormap(&map_v);
    ptx::prefetch_tensormap(&map_o);
  }
  if (warp == 13) {
    ptx::tmem_alloc(tmem_slot, 512);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;           // S0, S1 (128 columns each), O0, O1 (DP each)
  const uint32_t tmem_o = tmem + 256;

  bool ok = true;
  // the next item from i on whose source has keys
  auto with_keys = [&](int i, Item& t) {
    for (; i < p.items; i += gridDim.x) {
      t = item_of(p, i);
      if (t.len > 0) break;
    }
    return i;
  };
  // Whether the last block of an item has rows between its last key and the next multiple of 16, where its product ends, that TMA
  // has not zeroed.
  auto ragged = [&](const Item& t) { return (t.len & 15) != 0 && t.k0 + t.len < p.a.Tk; };
  if (warp >= 12) {
    ptx::registers_down<kOtherRegs>();
    if (warp == 12) {
      // ------------------------------ TMA producer -----------------------------------------------
      // The ring's first stage holds keys only; from then on values of a block and the keys of the next (or of the next item).
      if (lane == 0) {
        const uint64_t once = ptx::policy_evict_first(), again = ptx::policy_evict_last();
        int stage = 0; uint32_t phase = 0;
        uint32_t q_phase[2] = {0, 0};
        auto load = [&](const CUtensorMap* map, int off, int kh, int k0, int b) {
#pragma unroll
          for (int j = 0; j < DP / 64; ++j)
            ptx::tma_load_4d(ring + stage * L::stage + off + j * (kRows * 128), map, kv_full + stage, j * 64, kh, k0, b, again);
        };
        auto load_queries = [&](const Item& t, int half) {
          const Tile q = tile_of(p, t, half);
          if (!ptx::mbar_wait(q_empty + half, q_phase[half] ^ 1u, abort_flag)) { ok = false; return; }
          q_phase[half] ^= 1u;
          ptx::mbar_arrive_expect_tx(q_full + half, L::tile);
#pragma unroll
          for (int j = 0; j < DP / 64; ++j)
            ptx::tma_load_4d(smem + half * L::tile + j * (kRows * 128), &map_q, q_full + half, j * 64, q.h, q.q0, t.b, once);
        };
        Item t, n;
        int i = with_keys(blockIdx.x, t);
        if (i < p.items) {
          ptx::mbar_arrive_expect_tx(kv_full, L::tile);
          load(&map_k, L::tile, t.kh, t.k0, t.b);
          stage = 1;
          for (int half = 0; half < t.tiles && ok; ++half) load_queries(t, half);
        }
        while (i < p.items && ok) {
          const int ni = with_keys(i + gridDim.x, n);
          const bool more = ni < p.items;
          if (more)                            // the next item's queries are loaded only when this one's have been read for the last time
            for (int half = 0; half < n.tiles; ++half) {
              const Tile q = tile_of(p, n, half);
#pragma unroll
              for (int j = 0; j < DP / 64; ++j) ptx::tma_prefetch_4d(&map_q, j * 64, q.h, q.q0, n.b);
            }
          for (int k0 = 0; k0 < t.len; k0 += kRows) {
            const bool inner = k0 + kRows < t.len, keys = inner || more;
            if (!ptx::mbar_wait(kv_empty + stage, phase ^ 1u, abort_flag)) { ok = false; break; }
            ptx::mbar_arrive_expect_tx(kv_full + stage, keys ? L::stage : L::tile);
            load(&map_v, 0, t.kh, t.k0 + k0, t.b);
            if (inner) load(&map_k, L::tile, t.kh, t.k0 + k0 + kRows, t.b);
            else if (more) load(&map_k, L::tile, n.kh, n.k0, n.b);
            if (++stage == kStages) { stage = 0; phase ^= 1u; }
          }
          if (more)
            for (int half = 0; half < n.tiles && ok; ++half) load_queries(n, half);
          t = n;
          i = ni;
        }
      }
    } else if (warp == 13) {
      // ------------------------------ MMA issuer ---------------------------------------------------
      // One elected thread runs all of it.  Few MMAs queue up behind one another, so whatever this thread does between two of them
      // costs the tensor core: with a branch on lane 0 instead of elect.sync an MMA took 170 cycles to issue (64 in the tensor
      // core), whole-warp waits and a wait for each of keys and values cost a tenth of the kernel.
      if (ptx::elect_one()) {
        constexpr uint32_t idesc_s = ptx::make_idesc_bf16(kRows, kRows, false, false);
        constexpr uint32_t idesc_o = ptx::make_idesc_bf16(kRows, DP, false, true);
        int stage = 0; uint32_t phase = 0;
        uint32_t q_phase = 0, p_phase = 0, o_phase = 0;           // bit `half`
        auto wait = [&](uint64_t* bar, uint32_t parity) {
          if (ok) ok = ptx::mbar_wait(bar, parity & 1u, abort_flag);
          return ok;
        };
        // Scores of tile `half` against the keys in the ring's stage; `fresh`: the first of an item; `last`: the item's last.
        auto scores = [&](int half, bool fresh, bool last) {
          if (fresh) {
            if (!wait(q_full + half, q_phase >> half)) return;
            q_phase ^= 1u << half;
          }
          const uint32_t dq = ptx::smem_desc_low(smem + half * L::tile, 16), dk = ptx::smem_desc_low(ring + stage * L::stage + L::tile, 16);
#pragma unroll
          for (int k = 0; k < DP / 16; ++k) {
            const uint32_t off = (uint32_t)(k / 4 * (kRows * 128) + k % 4 * 32) >> 4;
            ptx::umma_bf16_low(tmem + half * kRows, dq + off, dk + off, idesc_s, k != 0 ? 1u : 0u);
          }
          ptx::umma_commit(s_full + half);
          if (last) ptx::umma_commit(q_empty + half);
        };
        Item t, n;
        int i = with_keys(blockIdx.x, t);
        if (i < p.items && wait(kv_full, 0)) {
          for (int half = 0; half < t.tiles && ok; ++half) scores(half, true, t.len <= kRows);
          ptx::umma_commit(kv_empty);
          stage = 1;
        }
        while (i < p.items && ok) {
          const int ni = with_keys(i + gridDim.x, n);
          const bool more = ni < p.items;
          const int blocks = ceil_div(t.len, kRows);
          for (int j = 0; j < blocks; ++j) {
            const int steps = min(kRows, (t.len - j * kRows + 15) & ~15) / 16;      // 16 keys each
            // the scores that follow: the next block's, or the next item's first
            const bool inner = j + 1 < blocks;
            const int s_tiles = inner ? t.tiles : more ? n.tiles : 0;
            const bool s_last = inner ? j + 2 == blocks : n.len <= kRows;
            if (!wait(kv_full + stage, phase)) break;
            if (!inner && ragged(t) && !wait(v_clean + stage, phase)) break;
            const uint32_t dv = ptx::smem_desc_low(ring + stage * L::stage, kRows * 128);
            for (int half = 0; half < 2 && ok; ++half) {
              if (half < t.tiles) {
                if (j == 0) {                        // the output before this one has left tensor memory
                  if (!wait(o_empty + half, (o_phase >> half) ^ 1u)) break;
                  o_phase ^= 1u << half;
                }
                if (!wait(p_full + half, p_phase >> half)) break;
                ptx::tc_fence_after_sync();
                p_phase ^= 1u << half;
                auto product = [&](int k) {
                  ptx::umma_bf16_ta(tmem_o + half * DP, tmem + half * kRows + k * 8, dv + (uint32_t)(k * 2048 >> 4), idesc_o, (j | k) != 0 ? 1u : 0u);
                };
                if (steps == kRows / 16) {
#pragma unroll
                  for (int k = 0; k < kRows / 16; ++k) product(k);
                } else {
                  for (int k = 0; k < steps; ++k) product(k);
                }
                if (!inner) ptx::umma_commit(o_full + half);
              }
              if (half < s_tiles) scores(half, !inner, s_last);
            }
            ptx::umma_commit(kv_empty + stage);
            if (++stage == kStages) { stage = 0; phase ^= 1u; }
          }
          t = n;
          i = ni;
        }
      }
    } else if (warp == 14) {
      // ------------------------------ zeroes what lies behind a source's last key ----------------------
      // It follows every stage, so that no phase of the barriers passes by unseen.
      int stage = 0; uint32_t phase = 0;
      auto follow = [&](int from, int to) {    // rows of V to zero
        if (!ptx::mbar_wait_all(kv_full + stage, phase, abort_flag)) { ok = false; return; }
        if (from < to) {
          unsigned char* sv = ring + stage * L::stage;
          for (int x = lane; x < (to - from) * (DP / 8); x += 32) {
            const int row = from + x / (DP / 8), c = x % (DP / 8);
            *reinterpret_cast<uint4*>(sv + c / 8 * (kRows * 128) + row * 128 + c % 8 * 16) = make_uint4(0, 0, 0, 0);
          }
          ptx::fence_proxy_async();
          __syncwarp();
        }
        if (lane == 0) {
          ptx::mbar_arrive(v_clean + stage);
          ptx::mbar_arrive(kv_empty + stage);
        }
        if (++stage == kStages) { stage = 0; phase ^= 1u; }
      };
      Item t;
      int i = with_keys(blockIdx.x, t);
      if (i < p.items) follow(0, 0);
      for (; i < p.items && ok; i = with_keys(i + gridDim.x, t))
        for (int k0 = 0; k0 < t.len && ok; k0 += kRows) {
          const int left = t.len - k0;
          const bool fix = left <= kRows && ragged(t);
          follow(fix ? left : 0, fix ? (left + 15) & ~15 : 0);
        }
    }
  } else if (warp >= 8) {
    // ------------------------------ output: one thread per row ---------------------------------------
    ptx::registers_down<kOutputRegs>();
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    unsigned char* stage = smem + L::out_off + (warp & 3) * 32 * 128;
    unsigned char* srow = stage + lane * 128;
    uint32_t phase = 0;                        // bit `half`
    for (int i = blockIdx.x; i < p.items && ok; i += gridDim.x) {
      const Item t = item_of(p, i);
      for (int half = 0; half < t.tiles && ok; ++half) {
        const Tile q = tile_of(p, t, half);
        const int r = (warp & 3) * 32 + lane;
        const bool in = r < q.rows, whole = p.parts == 1;
        int head = r;
        const int token = q.q0 + p.by_heads.split(head);
        head += q.h;
        float* lse = p.a.lse && in && whole ? p.a.lse + ((long long)t.b * p.a.H + head) * p.a.Tq + token : nullptr;
        const long long part_row = whole ? 0 : (((long long)t.part * p.a.B + t.b) * p.a.Tq + token) * p.a.H + head;
        float factor = 0.f;
        if (t.len > 0) {
          bool here = ptx::mbar_wait(stat_full + half, (phase >> half) & 1u, abort_flag) &&
                      ptx::mbar_wait(o_full + half, (phase >> half) & 1u, abort_flag);
          if (!__all_sync(0xffffffffu, here)) { ok = false; break; }
          phase ^= 1u << half;
          ptx::tc_fence_after_sync();
          const float sum = stat[half * 2 * kRows + r], top = stat[half * 2 * kRows + kRows + r];
          factor = 1.f / sum;
          if (lse) *lse = top * p.a.scale + logf(sum);
          if (!whole && in) p.part_lse[part_row] = fmaf(top, p.a.scale * kLog2e, log2f(sum));
        } else {
          if (lse) *lse = -INFINITY;
          if (!whole && in) p.part_lse[part_row] = -INFINITY;
        }
        if (!whole) {                          // a part's output, in fp32; nothing where it had no key
          if (t.len == 0) continue;
#pragma unroll
          for (int c = 0; c < DP / 32; ++c) {
            uint32_t o[32];
            ptx::tmem_ld_32x32(tmem_o + half * DP + c * 32 + lanes, o);
            ptx::tmem_ld_wait();
            if (c == DP / 32 - 1) {
              ptx::tc_fence_before_sync();
              __syncwarp();
              if (lane == 0) ptx::mbar_arrive(o_empty + half);
            }
#pragma unroll
            for (int x = 0; x < 32; x += 4)
              if (in && c * 32 + x < p.a.D)
                *reinterpret_cast<float4*>(p.part_o + part_row * p.a.D + c * 32 + x) =
                    make_float4(__uint_as_float(o[x]) * factor, __uint_as_float(o[x + 1]) * factor, __uint_as_float(o[x + 2]) * factor,
                                __uint_as_float(o[x + 3]) * factor);
          }
          continue;
        }
        // 64 columns at a time through the warp's staging rows
#pragma unroll
        for (int c = 0; c < DP / 64; ++c) {
          uint32_t w[32];
#pragma unroll
          for (int x = 0; x < 32; ++x) w[x] = 0;
          if (t.len > 0) {
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              uint32_t o[32];
              ptx::tmem_ld_32x32(tmem_o + half * DP + c * 64 + y * 32 + lanes, o);
              ptx::tmem_ld_wait();
#pragma unroll
              for (int x = 0; x < 16; ++x) {
                const __nv_bfloat162 b = __floats2bfloat162_rn(__uint_as_float(o[2 * x]) * factor, __uint_as_float(o[2 * x + 1]) * factor);
                w[y * 16 + x] = *reinterpret_cast<const uint32_t*>(&b);
              }
            }
            if (c == DP / 64 - 1) {
              ptx::tc_fence_before_sync();
              __syncwarp();
              if (lane == 0) ptx::mbar_arrive(o_empty + half);
            }
          }
          if (lane == 0) ptx::tma_store_wait_read();            // the store before has read the staging rows
          __syncwarp();
#pragma unroll
          for (int x = 0; x < 8; ++x)
            *reinterpret_cast<uint4*>(srow + ((x ^ (lane & 7)) * 16)) = make_uint4(w[4 * x], w[4 * x + 1], w[4 * x + 2], w[4 * x + 3]);
          ptx::fence_proxy_async();
          __syncwarp();
          const int token0 = q.q0 + p.by_heads.quotient((warp & 3) * 32);
          if (lane == 0 && token0 < p.a.Tq && c * 64 < p.a.D) {
            ptx::tma_store_4d(&map_o, stage, c * 64, q.h, token0, t.b);
            ptx::tma_store_commit();
          }
        }
      }
    }
    if (lane == 0) ptx::tma_store_wait_all();
  } else {
    // ------------------------------ softmax: one thread per row ----------------------------------
    ptx::registers_up<kSoftmaxRegs>();
    const int half = warp >> 2;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t t_s = tmem + half * kRows + lanes, t_o = tmem_o + half * DP + lanes;
    const float c = p.a.scale * kLog2e;
    uint32_t s_phase = 0, o_phase = 0;
    for (int i = blockIdx.x; i < p.items && ok; i += gridDim.x) {
      int len;
      {
        const Item t = item_of(p, i);
        len = half < t.tiles ? t.len : 0;
      }
      if (len == 0) continue;
      float top = -INFINITY, sum = 0.f;        // the maximum that the weights so far refer to, and their sum
      for (int k0 = 0; k0 < len; k0 += kRows) {
        if (!ptx::mbar_wait_all(s_full + half, s_phase, abort_flag)) { ok = false; break; }
        s_phase ^= 1u;
        ptx::tc_fence_after_sync();
        uint32_t s[kRows];
#pragma unroll
        for (int j = 0; j < 4; ++j) ptx::tmem_ld_32x32(t_s + j * 32, s + j * 32);
        ptx::tmem_ld_wait();
        const int left = len - k0;
        if (left < kRows) {
#pragma unroll
          for (int j = 0; j < kRows; ++j)
            if (j >= left) s[j] = 0xff800000u;
        }
        float m[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int j = 0; j < kRows; j += 2) m[j >> 1 & 3] = max3(m[j >> 1 & 3], __uint_as_float(s[j]), __uint_as_float(s[j + 1]));
        const float most = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
        if (k0 == 0) {
          top = most;
        } else {
          const bool grown = (most - top) * c > kSlack;
          if (__any_sync(0xffffffffu, grown)) {
            const float shrink = grown ? exp2_approx((top - most) * c) : 1.f;
            if (grown) top = most;
            sum *= shrink;
#pragma unroll
            for (int j = 0; j < DP / 16; ++j) {
              uint32_t o[16];
              ptx::tmem_ld_32x16(t_o + j * 16, o);
              ptx::tmem_ld_wait();
#pragma unroll
              for (int x = 0; x < 16; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * shrink);
              ptx::tmem_st_32x16(t_o + j * 16, o);
            }
          }
        }
        const f32x2 c2 = both(c), m2 = both(top == -INFINITY ? 0.f : -top * c);      // no score so far: no weight either, as 2^-inf
        f32x2 sum2[2] = {0, 0};
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          uint32_t w[16];
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const int at = h * 32 + 2 * j;
            const float2 x = unpair(fma2(pair(__uint_as_float(s[at]), __uint_as_float(s[at + 1])), c2, m2));
            const float e0 = exp2_approx(x.x), e1 = exp2_approx(x.y);
            sum2[j & 1] = add2(sum2[j & 1], pair(e0, e1));
            const __nv_bfloat162 b = __floats2bfloat162_rn(e0, e1);
            w[j] = *reinterpret_cast<const uint32_t*>(&b);
          }
          ptx::tmem_st_32x16(t_s + h * 16, w);
        }
        const float2 part = unpair(add2(sum2[0], sum2[1]));
        sum += part.x + part.y;
        ptx::tmem_st_wait();
        ptx::tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(p_full + half);
      }
      if (!ok) break;
      // the statistics of the item before have been read together with its output
      if (!ptx::mbar_wait_all(o_empty + half, o_phase ^ 1u, abort_flag)) { ok = false; break; }
      o_phase ^= 1u;
      const int r = threadIdx.x & 127;
      stat[half * 2 * kRows + r] = sum;
      stat[half * 2 * kRows + kRows + r] = top;
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(stat_full + half);
    }
  }

  // ------------------------------ teardown -------------------------------------------------------
  if (!ok) {
    *abort_flag = 1;
    set_device_status(p.a.status, GSHARD_ERR_TIMEOUT);
    const uint64_t t0 = ptx::globaltimer_ns();
    while (ptx::globaltimer_ns() - t0 < 2000000ull) { __nanosleep(1000); }
  }
  __syncwarp();
  ptx::tc_fence_before_sync();
  __syncthreads();
  if (warp == 13) {
    ptx::tc_fence_after_sync();
    ptx::tmem_dealloc(tmem, 512);
  }
}

// Heads of a tile: with all of a group's heads in it the keys are read once for them; the output warps' 32 rows are whole tokens.
int tile_heads(int group) { return 32 % group == 0 ? group : 1; }
int tiles_of(int Tq, int group) { return ceil_div(Tq, kRows / tile_heads(group)) * (group / tile_heads(group)); }
int items_of(int B, int Tq, int H, int Hkv) { return ceil_div(tiles_of(Tq, H / Hkv), 2) * Hkv * B; }

// in blocks of 128 keys
Parts source_parts(const AttentionArgs& a) { return parts_of(items_of(a.B, a.Tq, a.H, a.Hkv), ceil_div(a.Tk, kRows), 148); }

template <int DP>
int forward(const AttentionArgs& a, float* scratch, cudaStream_t st) {
  ForwardParams p;
  p.a = a;
  p.group = a.H / a.Hkv;
  p.heads = tile_heads(p.group);
  p.tokens = kRows / p.heads;
  p.q_tiles = ceil_div(a.Tq, p.tokens);
  p.list = tiles_of(a.Tq, a.H / a.Hkv);
  p.pairs = ceil_div(p.list, 2);
  const Parts parts = source_parts(a);
  p.parts = parts.parts;
  p.part_keys = parts.each * kRows;
  p.items = p.pairs * a.Hkv * a.B * p.parts;
  p.by_parts = Divisor(p.parts);
  p.by_pairs = Divisor(p.pairs);
  p.by_kv_heads = Divisor(a.Hkv);
  p.by_tiles = Divisor(p.q_tiles);
  p.by_heads = Divisor(p.heads);
  const long long rows = (long long)a.B * a.Tq * a.H;
  p.part_o = scratch;
  p.part_lse = scratch + p.parts * rows * a.D;
  CUtensorMap mq, mk, mv, mo;
  if (!make_token_map(&mq, a.q, a.D, a.H, a.Tq, a.B, a.q_stride, p.tokens, 64, p.heads) || !make_source_map(&mk, a, a.k, a.k_stride, kRows) ||
      !make_source_map(&mv, a, a.v, a.v_stride, kRows) || !make_token_map(&mo, a.o, a.D, a.H, a.Tq, a.B, (long long)a.H * a.D, 32 / p.heads, 64, p.heads))
    return GSHARD_ERR_CUDA;
  auto kernel = attention_umma_forward_kernel<DP>;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Layout<DP>::bytes) != cudaSuccess) {
    cudaGetLastError();
    return GSHARD_ERR_CUDA;
  }
  kernel<<<std::min(p.items, device_sms()), kThreads, Layout<DP>::bytes, st>>>(mq, mk, mv, mo, p);
  count_launch();
  if (cudaGetLastError() != cudaSuccess) return GSHARD_ERR_CUDA;
  return p.parts > 1 ? launch_join_outputs(a, true, p.part_o, p.part_lse, p.parts, st) : GSHARD_OK;
}

}  // namespace

size_t attention_umma_forward_floats(const AttentionArgs& a) {
  const int parts = source_parts(a).parts;
  return parts > 1 ? (size_t)parts * a.B * a.Tq * a.H * (a.D + 1) : 0;
}

int launch_attention_umma_forward(const AttentionArgs& a, float* scratch, cudaStream_t st) {
  return a.D <= 64 ? forward<64>(a, scratch, st) : forward<128>(a, scratch, st);
}

}  // namespace gshard
