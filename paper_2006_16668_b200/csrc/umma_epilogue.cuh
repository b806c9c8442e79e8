// Epilogue of the grouped tcgen05 GEMMs (one-SM and CTA-pair kernels): accumulator rows out of tensor
// memory, ReLU / mask, conversion, staging in swizzled shared memory, 128-byte row stores.  `P` is
// the kernel's parameter struct (C, mask, rows, cols, c_ld, c_bs, out_f32, relu).
#pragma once
#include "activation.cuh"
#include "kernels.cuh"
#include "sm100_ptx.cuh"

namespace gshard {
namespace umma_epi {

constexpr int kTileRows = 128;
constexpr int kStgRowBytes = 128;           // staging: 32 rows x 128 bytes per warp
constexpr int kStgWarpBytes = 32 * kStgRowBytes;

struct TileCoord { int mt, nt, b; };

// Ragged batches (compacted expert rows).  Problem b owns the row tiles [tile_base[b], tile_base[b+1]) of
// a device-side prefix array with batch + 1 entries, and tile_problem[r] names the problem that owns
// row tile r, so a tile index is decoded with three loads and no search; the callers decode the NEXT
// tile before they work on the current one, which hides those loads.  Within a problem the row tiles
// run fastest: they share the B tile.
template <typename P>
__device__ __forceinline__ TileCoord decode_ragged(const P& p, int tile) {
  TileCoord t;
  t.b = __ldg(p.tile_problem + tile / p.n_tiles);
  const int first = __ldg(p.tile_base + t.b);
  const int m_b = __ldg(p.tile_base + t.b + 1) - first;
  const int i = tile - first * p.n_tiles;
  t.mt = i % m_b; t.nt = i / m_b;
  return t;
}

// Products of operands that are sums of bf16 planes.  An fp32 value is hi + mid + lo, each the next 8 bits; of the nine
// products the six that reach 2^-16 of the largest are added, small ones first, plane numbers in nibbles per pass.
constexpr int kPasses3 = 6, kPassA3 = 0x001012, kPassB3 = 0x010210;      // lo hi, mid mid, hi lo, mid hi, hi mid, hi hi
__host__ __device__ __forceinline__ int plane_of(int table, int pass) { return (table >> (4 * pass)) & 0xf; }

// The tensor core truncates its running sum at every step (16 products), so an fp32-accurate product must not stay in
// it for long: a run of at most 4 k-blocks (256 deep) of the hi hi pass, after which the epilogue warps add the run to
// fp32 sums in their registers, rounding to nearest; the other passes, 2^-8 of it, in runs of 64 k-blocks.  16-bit
// operands with fp32 output have the one pass.  (One
// accumulation over 1024: 1e-6 relative error, over 8192: 8e-6; in runs 3e-7 at any length.)
constexpr int kHiRun = 4, kLowRun = 64;
__device__ __forceinline__ int low_runs(int k_blocks, int passes) { return ((passes - 1) * k_blocks + kLowRun - 1) / kLowRun; }
__device__ __forceinline__ int all_runs(int k_blocks, int passes) {
  return low_runs(k_blocks, passes) + (k_blocks + kHiRun - 1) / kHiRun;
}
__device__ __forceinline__ int run_length(int run, int k_blocks, int passes) {
  const int low = low_runs(k_blocks, passes);
  return run < low ? min(kLowRun, (passes - 1) * k_blocks - run * kLowRun) : min(kHiRun, k_blocks - (run - low) * kHiRun);
}

// Writes a warp's staged 32 rows x 128 bytes to C: lane l handles 16-byte piece (l & 7) of rows
// 4*i + (l >> 3); pieces beyond the matrix edge are skipped (cols is a multiple of the piece width).
// Whether the output rows should be kept in L2 (they are re-read soon by the same launch).  A kernel
// whose parameter struct wants that overloads this for its struct.
template <typename P>
__device__ __forceinline__ bool epi_keep_in_l2(const P&) { return false; }

template <typename P>
__device__ __forceinline__ void flush_rows(const unsigned char* stg, const P& p, int b, int row0, int col0,
                                           int lane) {
  __syncwarp();
  const bool keep = epi_keep_in_l2(p);
  const uint64_t pol = keep ? ptx::policy_evict_last() : 0ull;
  const int esz = p.out_f32 ? 4 : 2;
  const int piece = lane & 7;
  const int col = col0 + piece * (16 / esz);
  unsigned char* cbase = reinterpret_cast<unsigned char*>(p.C) + ((long long)b * p.c_bs + col) * esz;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = 4 * i + (lane >> 3);
    const int row = row0 + r;
    if (row < p.rows && col < p.cols) {
      const uint4 val = *reinterpret_cast<const uint4*>(stg + r * kStgRowBytes + ((piece ^ (r & 7)) * 16));
      uint4* dst = reinterpret_cast<uint4*>(cbase + (long long)row * p.c_ld * esz);
      if (keep)
        asm volatile("st.global.L2::cache_hint.v4.b32 [%0], {%1, %2, %3, %4}, %5;" ::"l"(dst), "r"(val.x), "r"(val.y),
                     "r"(val.z), "r"(val.w), "l"(pol)
                     : "memory");
      else
        *dst = val;
    }
  }
  __syncwarp();
}

// The same block through the TMA unit: the warp's 32 staged rows x 128 bytes (already in the 128-byte
// swizzle a tensor map expects, the staging block being 1024-byte aligned) leave as one bulk tensor
// store; rows and columns beyond the matrix are clipped by the tensor map.  Compared with flush_rows
// this takes the re-read of the staging rows and the global stores off the load/store pipe.  The
// staging block may be rewritten only after store_wait().
__device__ __forceinline__ void flush_rows_tma(const unsigned char* stg, const CUtensorMap* map_c, int b, int row0,
                                               int col0, int lane) {
  ptx::fence_proxy_async();          // this lane's staged bytes visible to the async proxy
  __syncwarp();
  if (lane == 0) {
    ptx::tma_store_3d(map_c, stg, col0, row0, b);
    ptx::tma_store_commit();
  }
}
__device__ __forceinline__ void store_wait(int lane) {
  if (lane == 0) ptx::tma_store_wait_read();
  __syncwarp();
}

// ReLU / mask on one 32-column chunk of this thread's row, then into the staging row (XOR-swizzled
// 16-byte pieces: conflict-free for the row-wise writes here and the piece-wise reads of the flush).
// mword: with MASK, bit i set = keep column i of the chunk.
template <bool MASK, typename P>
__device__ __forceinline__ void process_chunk(const uint32_t* r, const P& p, unsigned char* srow, int lane,
                                              int piece0, uint32_t mword) {
  float v[32];
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    v[i] = __uint_as_float(r[i]);
    if (p.relu) v[i] = fmaxf(v[i], 0.f);
    if (MASK && !((mword >> i) & 1u)) v[i] = 0.f;
  }
  if (p.out_f32) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      *reinterpret_cast<float4*>(srow + (((piece0 + i) ^ (lane & 7)) * 16)) =
          make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const __nv_bfloat162 pr = __floats2bfloat162_rn(v[8 * i + 2 * j], v[8 * i + 2 * j + 1]);
        w[j] = *reinterpret_cast<const uint32_t*>(&pr);
      }
      *reinterpret_cast<uint4*>(srow + (((piece0 + i) ^ (lane & 7)) * 16)) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}

// First column of round c of this warp's half of the tile.
template <int BN>
__device__ __forceinline__ int round_col0(const TileCoord& t, int half, int c) {
  return t.nt * BN + half * (BN / 2) + c * 64;
}

// Bit i of the result: accumulator value i of the chunk is positive (the ReLU passes it).
__device__ __forceinline__ uint32_t positive_bits(const uint32_t* r) {
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 32; ++i) w |= (__uint_as_float(r[i]) > 0.f ? 1u : 0u) << i;
  return w;
}

// One epilogue warp's share of a finished 128 x BN accumulator whose first row is tile_row0: lane
// quarter q, column half `half`.  map_c: tensor map of C for bulk stores, or nullptr for plain 16-byte
// stores.  With MASK (bf16 output only) the output is zeroed where the bit of p.mask_bits
// ([batch][rows][cols/32] words, bit = column mod 32) is clear; the two words of a thread's row and
// round are fetched while the accumulator load is in flight.  With p.mask_bits_out the same layout is
// WRITTEN: bit = accumulator value positive (the ReLU mask the backward pass needs).
template <int BN, bool MASK, typename P>
__device__ __forceinline__ void epilogue_tile(const P& p, const CUtensorMap* map_c, const TileCoord& t, int tile_row0,
                                              uint32_t tmem_acc, int q, int half, unsigned char* stg, int lane) {
  constexpr int kHalfCols = BN / 2;
  unsigned char* srow = stg + lane * kStgRowBytes;
  const int row0 = tile_row0 + q * 32;
  const int row = row0 + lane;
  const long long word_row = ((long long)t.b * p.rows + row) * (p.cols >> 5);
  const uint32_t t_acc = tmem_acc + (uint32_t)(half * kHalfCols) + ((uint32_t)(q * 32) << 16);
#pragma unroll 1
  for (int c = 0; c < kHalfCols / 64; ++c) {     // 64 columns per round: two TMEM loads in flight
    const int col0 = round_col0<BN>(t, half, c);
    if (col0 >= p.cols) break;                   // uniform over the warp
    uint32_t r0[32], r1[32];
    ptx::tmem_ld_32x32(t_acc + (uint32_t)(c * 64), r0);
    ptx::tmem_ld_32x32(t_acc + (uint32_t)(c * 64 + 32), r1);
    uint32_t m0 = 0, m1 = 0;
    if (MASK && row < p.rows) {
      m0 = __ldg(p.mask_bits + word_row + (col0 >> 5));
      if (col0 + 32 < p.cols) m1 = __ldg(p.mask_bits + word_row + (col0 >> 5) + 1);
    }
    if (map_c) store_wait(lane);                 // the previous bulk store has read the staging block
    ptx::tmem_ld_wait();
    if (p.mask_bits_out && row < p.rows) {
      p.mask_bits_out[word_row + (col0 >> 5)] = positive_bits(r0);
      if (col0 + 32 < p.cols) p.mask_bits_out[word_row + (col0 >> 5) + 1] = positive_bits(r1);
    }
    if (p.out_f32) {                             // 32 fp32 columns = one 128-byte staging row
      process_chunk<MASK>(r0, p, srow, lane, 0, m0);
      if (map_c) { flush_rows_tma(stg, map_c, t.b, row0, col0, lane); store_wait(lane); }
      else flush_rows(stg, p, t.b, row0, col0, lane);
      process_chunk<MASK>(r1, p, srow, lane, 0, m1);
      if (map_c) flush_rows_tma(stg, map_c, t.b, row0, col0 + 32, lane);
      else flush_rows(stg, p, t.b, row0, col0 + 32, lane);
    } else {                                     // 64 bf16 columns = one 128-byte staging row
      process_chunk<MASK>(r0, p, srow, lane, 0, m0);
      process_chunk<MASK>(r1, p, srow, lane, 4, m1);
      if (map_c) flush_rows_tma(stg, map_c, t.b, row0, col0, lane);
      else flush_rows(stg, p, t.b, row0, col0, lane);
    }
  }
}

// The linear operator's epilogue: pre = acc + bias, C = act(pre) + residual, and pre itself where the caller
// keeps it.  Same share of the tile and same bulk tensor stores as above.  64 columns per round stay in
// registers, so that pre and C can leave one after the other through the one staging block; the residual's 64
// columns of the thread's row are fetched ahead.  All of it in fp32, rounded once per output.
// One round: 64 columns from col0 of this thread's row, in r.  WAIT: tensor-memory loads into r are still in flight.
// F32: the output is known to be fp32.
template <bool WAIT, bool F32, typename P>
__device__ __forceinline__ void linear_round(const P& p, const CUtensorMap* map_c, const CUtensorMap* map_pre, int b, int row0,
                                             int col0, uint32_t (*r)[32], unsigned char* stg, int lane) {
  unsigned char* srow = stg + lane * kStgRowBytes;
  const int row = row0 + lane;
  const bool f32 = F32 || p.out_f32;
  struct Plain { int relu, out_f32; } plain{0, f32};
  uint4 res[8];                                  // bf16 residual: 64 columns (an fp32 one is read below)
  const bool has_res = p.lin.residual != nullptr && row < p.rows;
  const long long off = (long long)row * p.c_ld + col0;
  if (has_res && !f32) {
    const uint4* src = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.lin.residual) + off);
#pragma unroll
    for (int i = 0; i < 8; ++i) res[i] = col0 + 8 * i < p.cols ? src[i] : make_uint4(0, 0, 0, 0);
  }
  store_wait(lane);                              // the previous bulk store has read the staging block
  if (WAIT) ptx::tmem_ld_wait();
  if (p.lin.bias) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 32; i += 4) {
        const int col = col0 + 32 * h + i;
        if (col < p.cols) {                    // cols is a multiple of 8
          const float4 b = __ldg(reinterpret_cast<const float4*>(p.lin.bias + col));
          r[h][i] = __float_as_uint(__uint_as_float(r[h][i]) + b.x);
          r[h][i + 1] = __float_as_uint(__uint_as_float(r[h][i + 1]) + b.y);
          r[h][i + 2] = __float_as_uint(__uint_as_float(r[h][i + 2]) + b.z);
          r[h][i + 3] = __float_as_uint(__uint_as_float(r[h][i + 3]) + b.w);
        }
      }
  }
  if (p.lin.pre) {
    process_chunk<false>(r[0], plain, srow, lane, 0, 0);
    if (f32) {
      flush_rows_tma(stg, map_pre, b, row0, col0, lane);
      store_wait(lane);
      process_chunk<false>(r[1], plain, srow, lane, 0, 0);
      if (col0 + 32 < p.cols) flush_rows_tma(stg, map_pre, b, row0, col0 + 32, lane);
    } else {
      process_chunk<false>(r[1], plain, srow, lane, 4, 0);
      flush_rows_tma(stg, map_pre, b, row0, col0, lane);
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (f32) activate<32, false>(r[h], p.lin.act);
    else activate<32, true>(r[h], p.lin.act);
    if (has_res) {
      if (f32) {
        const float4* src = reinterpret_cast<const float4*>(static_cast<const float*>(p.lin.residual) + off + 32 * h);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (col0 + 32 * h + 4 * i < p.cols) {
            const float4 f = src[i];
            r[h][4 * i] = __float_as_uint(__uint_as_float(r[h][4 * i]) + f.x);
            r[h][4 * i + 1] = __float_as_uint(__uint_as_float(r[h][4 * i + 1]) + f.y);
            r[h][4 * i + 2] = __float_as_uint(__uint_as_float(r[h][4 * i + 2]) + f.z);
            r[h][4 * i + 3] = __float_as_uint(__uint_as_float(r[h][4 * i + 3]) + f.w);
          }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float f[8];
          Vec16<__nv_bfloat16>::load(res[4 * h + i], f);
#pragma unroll
          for (int j = 0; j < 8; ++j) r[h][8 * i + j] = __float_as_uint(__uint_as_float(r[h][8 * i + j]) + f[j]);
        }
      }
    }
  }
  if (p.lin.pre) store_wait(lane);
  process_chunk<false>(r[0], plain, srow, lane, 0, 0);
  if (f32) {
    flush_rows_tma(stg, map_c, b, row0, col0, lane);
    store_wait(lane);
    process_chunk<false>(r[1], plain, srow, lane, 0, 0);
    if (col0 + 32 < p.cols) flush_rows_tma(stg, map_c, b, row0, col0 + 32, lane);
  } else {
    process_chunk<false>(r[1], plain, srow, lane, 4, 0);
    flush_rows_tma(stg, map_c, b, row0, col0, lane);
  }
}

template <int BN, typename P>
__device__ __forceinline__ void epilogue_linear_tile(const P& p, const CUtensorMap* map_c, const CUtensorMap* map_pre,
                                                     const TileCoord& t, int tile_row0, uint32_t tmem_acc, int q, int half,
                                                     unsigned char* stg, int lane) {
  constexpr int kHalfCols = BN / 2;
  const uint32_t t_acc = tmem_acc + (uint32_t)(half * kHalfCols) + ((uint32_t)(q * 32) << 16);
#pragma unroll 1
  for (int c = 0; c < kHalfCols / 64; ++c) {
    const int col0 = round_col0<BN>(t, half, c);
    if (col0 >= p.cols) break;                   // uniform over the warp
    uint32_t r[2][32];
    ptx::tmem_ld_32x32(t_acc + (uint32_t)(c * 64), r[0]);
    ptx::tmem_ld_32x32(t_acc + (uint32_t)(c * 64 + 32), r[1]);
    linear_round<true, false>(p, map_c, map_pre, t.b, tile_row0 + q * 32, col0, r, stg, lane);
  }
}

// sums (+)= this warp's share of a finished run: 32 rows x BN / 2 columns, one row per lane, as fp32 bits.
// GATED: a quarter of the columns of either factor instead.
template <int BN, bool GATED = false>
__device__ __forceinline__ void add_run(uint32_t (*sums)[32], uint32_t tmem_acc, int q, int half, bool first) {
  const uint32_t t_acc = tmem_acc + (uint32_t)(half * (GATED ? BN / 4 : BN / 2)) + ((uint32_t)(q * 32) << 16);
#pragma unroll
  for (int c = 0; c < BN / 32; ++c) {              // 16 columns at a time: the sums take most of the registers
    uint32_t r[16];
    ptx::tmem_ld_32x16(t_acc + (uint32_t)(c * 16 + (GATED && c >= BN / 64 ? BN / 4 : 0)), r);
    ptx::tmem_ld_wait();
    uint32_t* s = &sums[c / 2][c % 2 * 16];
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = __float_as_uint(__uint_as_float(r[i]) + (first ? 0.f : __uint_as_float(s[i])));
  }
}
template <int BN, typename P>
__device__ __forceinline__ void epilogue_linear_sums(const P& p, const CUtensorMap* map_c, const CUtensorMap* map_pre,
                                                     const TileCoord& t, int tile_row0, uint32_t (*sums)[32], int q, int half,
                                                     unsigned char* stg, int lane) {
#pragma unroll
  for (int c = 0; c < BN / 128; ++c) {
    const int col0 = round_col0<BN>(t, half, c);
    if (col0 < p.cols) linear_round<false, true>(p, map_c, map_pre, t.b, tile_row0 + q * 32, col0, sums + 2 * c, stg, lane);
  }
}

// The gated linear operator's epilogue: the accumulator's first half of columns are gate columns, its second half the
// same columns of the other factor; h = act(gate) up, and both factors themselves where the caller keeps them (map_pre: batch 0
// the gates, 1 the other factors).  A round is 64 columns of a warp's 32 rows.
template <bool F32, typename P>
__device__ __forceinline__ void gated_round(const P& p, const CUtensorMap* map_c, const CUtensorMap* map_pre, int row0, int col0,
                                            uint32_t (*g)[32], uint32_t (*u)[32], unsigned char* stg, int lane) {
  unsigned char* srow = stg + lane * kStgRowBytes;
  struct Plain { int relu, out_f32; } plain{0, F32};
  auto put = [&](uint32_t (*r)[32], const CUtensorMap* map, int b) {       // 64 columns through the staging rows
    store_wait(lane);                            // the previous bulk store has read them
    process_chunk<false>(r[0], plain, srow, lane, 0, 0);
    if (F32) {
      flush_rows_tma(stg, map, b, row0, col0, lane);
      store_wait(lane);
      process_chunk<false>(r[1], plain, srow, lane, 0, 0);
      if (col0 + 32 < p.cols) flush_rows_tma(stg, map, b, row0, col0 + 32, lane);
    } else {
      process_chunk<false>(r[1], plain, srow, lane, 4, 0);
      flush_rows_tma(stg, map, b, row0, col0, lane);
    }
  };
  if (p.lin.pre) {
    put(g, map_pre, 0);
    put(u, map_pre, 1);
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    activate<32, !F32>(g[h], p.lin.act);
#pragma unroll
    for (int i = 0; i < 32; ++i) g[h][i] = __float_as_uint(__uint_as_float(g[h][i]) * __uint_as_float(u[h][i]));
  }
  put(g, map_c, 0);
}

// One epilogue warp's share of a finished tile: column half `half` of both factors.
template <int BN, typename P>
__device__ __forceinline__ void epilogue_gated_tile(const P& p, const CUtensorMap* map_c, const CUtensorMap* map_pre, const TileCoord& t,
                                                    int tile_row0, uint32_t tmem_acc, int q, int half, unsigned char* stg, int lane) {
  const int col0 = t.nt * (BN / 2) + half * (BN / 4);
  static_assert(BN / 4 == 64, "one round per warp");
  if (col0 >= p.cols) return;                    // uniform over the warp
  const uint32_t t_acc = tmem_acc + (uint32_t)(half * (BN / 4)) + ((uint32_t)(q * 32) << 16);
  uint32_t g[2][32], u[2][32];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    ptx::tmem_ld_32x32(t_acc + h * 32, g[h]);
    ptx::tmem_ld_32x32(t_acc + BN / 2 + h * 32, u[h]);
  }
  ptx::tmem_ld_wait();
  gated_round<false>(p, map_c, map_pre, tile_row0 + q * 32, col0, g, u, stg, lane);
}

// After a warp's last tile: its bulk stores have left shared memory and reached global memory.
__device__ __forceinline__ void epilogue_finish(const CUtensorMap* map_c, int lane) {
  if (map_c && lane == 0) ptx::tma_store_wait_all();
  __syncwarp();
}

}  // namespace umma_epi
}  // namespace gshard
