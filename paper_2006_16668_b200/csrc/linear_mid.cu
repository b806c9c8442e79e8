// The linear operator's matrix products whose output tiles fit the multiprocessors at once (decoding steps of a batch,
// short sequences): y [rows, cols] = A . B on the tensor cores in ONE launch.  Here time is not work but what happens
// once: launches, filling the pipeline, the epilogue's round trips.  So
//   * no persistent loop and no tile list: a CTA computes one 128 x BN tile, the narrowest BN (64 or 128) with which all
//     tiles run at once, which spreads B over as many multiprocessors as can read it;
//   * where tiles are few the contraction is cut among the 2 or 4 CTAs of a cluster.  Each owns a share of the tile's
//     rows; every CTA sends its fp32 sums of those rows to the owner's shared memory, and the owner adds them in the
//     order of the ranks (the same bits every time).  One cluster barrier, no partial product through memory, no second
//     kernel;
//   * a stage is 128 deep: a k-block costs the issuing thread some 190 cycles for its barriers whatever the tile
//     holds, and each MMA 35;
//   * the status word is cleared by the first CTA instead of a memset before the launch (3 us less).  A CTA reports only
//     after a wait of two seconds ran out, long after the first CTA of a grid whose CTAs all run at once began.
// fp32 operands come as three bf16 planes (linear.cu).  Warp 0 feeds TMA loads, warp 1 issues the MMAs, then all eight warps take the accumulator out of tensor memory.
#include <cuda.h>

#include <algorithm>

#include "activation.cuh"
#include "linear.cuh"
#include "pack.cuh"
#include "sm100_ptx.cuh"
#include "tensor_map.cuh"
#include "umma_epilogue.cuh"

namespace gshard {

namespace {

constexpr int kMidThreads = 256;
constexpr int kMidRows = 128, kMidDepth = 128;         // rows of a tile, depth of a k-block (two swizzled 64-deep halves)
constexpr int kMidBox = 64 * kMidDepth * 2;            // one box of an MN-major operand: 64 columns, the whole depth
constexpr int kMidMaxStages = 12;
constexpr int kMidBarBytes = 1024;                     // barriers, before the stages
constexpr int kMidSmem = 226 * 1024;                   // used at most
constexpr int kMidAlone = 120 * 1024;                  // asked for at least: more than half of a multiprocessor's
constexpr int kMidSms = 148;

struct MidArgs {
  void* y;
  LinearEpilogue lin;
  int* status;
  int clear_status;
  int rows, cols, k_blocks, run;        // run: k-blocks per CTA of the cluster
  int passes, pass_a, pass_b;           // operands in planes: every k-block once per product (plane numbers in nibbles)
  int a_once, b_once;                   // operand read by one CTA only
  int a_half, stages;                   // bytes of A's rows in half a stage
};

// fp32 output: the tensor core truncates its running sum at every step, so the leading product stays in an accumulator for
// two k-blocks (256 deep) only and the epilogue adds the accumulators, rounding to nearest.  With operands in three planes
// the five small products (2^-8 of it) come first, in two accumulators.  All of it lies in tensor memory at once.
constexpr int kMidRunAccs = 8, kMidRun = 2;
__device__ __forceinline__ int run_of(int it, int blocks, int passes) {
  const int low = (passes - 1) * blocks;
  if (it < low) return 2 * it >= low ? 1 : 0;
  return (low ? 2 : 0) + (it - low) / kMidRun;
}
// K-blocks per CTA up to which this is the faster path.  Three planes are six products of each k-block: 512 rows of
// 1024 -> 1024 (4 k-blocks) 22.1 to 18.0 us, 256 rows of 3000 -> 1024 (6) 26.9 to 28.7, 64 of 4096 -> 1024 (8) equal.  One
// product with fp32 output: what tensor memory holds (16), 256 rows of 3000 -> 1024 13.9 to 9.6.
int most_k_blocks(int passes, bool out_f32) {
  if (out_f32) return passes > 1 ? 4 : kMidRunAccs * kMidRun;
  return 64 / passes;
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void st_peer(uint32_t addr, float a, float b, float c, float d) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(a), "f"(b), "f"(c), "f"(d) : "memory");
}

template <bool A_K, bool B_K, int BN, int SPLITS, typename TY>
__global__ void __launch_bounds__(kMidThreads, 1)
linear_mid_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const MidArgs p) {
  constexpr bool RUNS = sizeof(TY) == 4;
  constexpr int kAccs = RUNS ? kMidRunAccs : 1;
  constexpr int kBBytes = BN * kMidDepth * 2, kLd = BN + 4;      // floats per row of sums: rows start in different banks
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* full = reinterpret_cast<uint64_t*>(smem);
  uint64_t* empty = full + kMidMaxStages;
  uint64_t* acc_full = empty + kMidMaxStages;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_full + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  smem += kMidBarBytes;
  const int stage_bytes = 2 * p.a_half + kBBytes, stages = p.stages;
  // one CTA alone puts its sums over the stages, which are free by then; those of a cluster may still be loading
  float* sums = reinterpret_cast<float*>(smem + (SPLITS > 1 ? stages * stage_bytes : 0));
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int rank = SPLITS > 1 ? blockIdx.x : 0;        // the cluster spans grid.x
  const int row0 = blockIdx.z * kMidRows, col0 = blockIdx.y * BN;

  if (tid == 0) {
    if (p.clear_status && blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0) *p.status = 0;
    ptx::prefetch_tensormap(&map_a);
    ptx::prefetch_tensormap(&map_b);
    for (int s = 0; s < stages; ++s) { ptx::mbar_init(full + s, 1); ptx::mbar_init(empty + s, 1); }
    ptx::mbar_init(acc_full, 1);
    *abort_flag = 0;
    ptx::fence_mbar_init();
  }
  if (warp == 1) {
    ptx::tmem_alloc(tmem_slot, kAccs * BN);
    ptx::tmem_relinquish();
  }
  // what the epilogue adds to every row of this thread's four columns
  constexpr int kQuads = BN / 4;
  const int col = col0 + tid % kQuads * 4;
  const bool in = col < p.cols;                        // cols is a multiple of 8
  float4 bias = make_float4(0.f, 0.f, 0.f, 0.f);
  if (p.lin.bias && in) bias = __ldg(reinterpret_cast<const float4*>(p.lin.bias + col));
  __syncwarp();
  if (SPLITS > 1) cluster_arrive();                    // waited for before the first store into another CTA
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;

  const int kb0 = rank * p.run, blocks = min(p.run, p.k_blocks - kb0), iters = blocks * p.passes;
  bool ok = true;
  // A lane elected once per loop: what it issues goes to the TMA and tensor units from values that the compiler knows
  // to be one thread's (an MMA issued by lane 0 of a diverged warp took 70 cycles).
  if (warp == 0) {
    if (ptx::elect_one()) {
      const uint64_t pol_a = p.a_once ? ptx::policy_evict_first() : ptx::policy_evict_last();
      const uint64_t pol_b = p.b_once ? ptx::policy_evict_first() : ptx::policy_evict_last();
      int stage = 0; uint32_t phase = 0;
      for (int it = 0, kb = 0, pass = 0; it < iters; ++it) {
        const int pa = umma_epi::plane_of(p.pass_a, pass), pb = umma_epi::plane_of(p.pass_b, pass);
        if (!ptx::mbar_wait(empty + stage, phase ^ 1u, abort_flag)) { ok = false; break; }
        unsigned char* sa = smem + stage * stage_bytes;
        unsigned char* sb = sa + 2 * p.a_half;
        ptx::mbar_arrive_expect_tx(full + stage, (uint32_t)stage_bytes);
        const int k0 = (kb0 + kb) * kMidDepth;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if (A_K) ptx::tma_load_3d(sa + j * p.a_half, &map_a, full + stage, k0 + j * 64, row0, pa, pol_a);
          else ptx::tma_load_3d(sa + j * kMidBox, &map_a, full + stage, row0 + j * 64, k0, pa, pol_a);
        }
#pragma unroll
        for (int j = 0; j < (B_K ? 2 : BN / 64); ++j) {
          if (B_K) ptx::tma_load_3d(sb + j * (kBBytes / 2), &map_b, full + stage, k0 + j * 64, col0, pb, pol_b);
          else ptx::tma_load_3d(sb + j * kMidBox, &map_b, full + stage, col0 + j * 64, k0, pb, pol_b);
        }
        if (++kb == blocks) { kb = 0; ++pass; }
        if (++stage == stages) { stage = 0; phase ^= 1u; }
      }
    }
  } else if (warp == 1) {
    if (ptx::elect_one()) {
      constexpr uint32_t idesc = ptx::make_idesc_bf16(kMidRows, BN, !A_K, !B_K);
      int stage = 0; uint32_t phase = 0;
      int prev = -1;
      for (int it = 0; it < iters; ++it) {
        const int acc = RUNS ? run_of(it, blocks, p.passes) : 0;
        const bool more = acc == prev;                 // than the accumulator's first k-block
        prev = acc;
        if (!ptx::mbar_wait(full + stage, phase, abort_flag)) { ok = false; break; }
        ptx::tc_fence_after_sync();
        const uint32_t sa = ptx::smem_u32(smem + stage * stage_bytes), sb = sa + 2 * p.a_half;
#pragma unroll
        for (int k = 0; k < kMidDepth / 16; ++k) {
          const uint64_t da = A_K ? ptx::make_smem_desc(sa + k / 4 * p.a_half + k % 4 * 32, 16, 1024)
                                  : ptx::make_smem_desc(sa + k * 2048, kMidBox, 1024);
          const uint64_t db = B_K ? ptx::make_smem_desc(sb + k / 4 * (kBBytes / 2) + k % 4 * 32, 16, 1024)
                                  : ptx::make_smem_desc(sb + k * 2048, kMidBox, 1024);
          ptx::umma_bf16(tmem + (uint32_t)(acc * BN), da, db, idesc, more || k != 0 ? 1u : 0u);
        }
        ptx::umma_commit(empty + stage);
        if (++stage == stages) { stage = 0; phase ^= 1u; }
      }
      if (ok) ptx::umma_commit(acc_full);
    }
  }
  __syncwarp();
  if (!ptx::mbar_wait_warp(acc_full, 0, abort_flag, lane)) ok = false;
  if (!ok) { *abort_flag = 1; set_device_status(p.status, GSHARD_ERR_TIMEOUT); }
  ptx::tc_fence_after_sync();
  __syncthreads();
  const bool failed = *abort_flag != 0;
  __syncwarp();
  if (SPLITS > 1) cluster_wait();                      // every CTA of the cluster runs: its shared memory may be written
  const int valid = min(kMidRows, p.rows - row0);
  const int share = (valid + SPLITS - 1) / SPLITS;     // rows that a CTA of the cluster owns
  if (failed) {
    // copies and MMAs in flight get a bounded time to land before shared and tensor memory are released
    const uint64_t t0 = ptx::globaltimer_ns();
    while (ptx::globaltimer_ns() - t0 < 2000000ull) { __nanosleep(1000); }
  } else {
    const int q = warp & 3, half = warp >> 2;          // a warp reads its quarter of the rows, half of the columns
    if (q * 32 < valid) {
      const int r = q * 32 + lane, owner = r / share;
      uint32_t dst = ptx::smem_u32(sums + (rank * share + r - owner * share) * kLd + half * (BN / 2));
      if (SPLITS > 1) dst = ptx::map_to_cta(dst, r < valid ? owner : rank);
      const uint32_t src = tmem + (uint32_t)(half * (BN / 2)) + ((uint32_t)(q * 32) << 16);
#pragma unroll
      for (int c = 0; c < BN / 2; c += 32) {
        uint32_t v[32];
        ptx::tmem_ld_32x32(src + (uint32_t)c, v);
        ptx::tmem_ld_wait();
        if (RUNS) {
          const int accs = run_of(iters - 1, blocks, p.passes) + 1;
#pragma unroll 1
          for (int a = 1; a < accs; ++a) {             // small terms first
            uint32_t more[32];
            ptx::tmem_ld_32x32(src + (uint32_t)(a * BN + c), more);
            ptx::tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) + __uint_as_float(more[i]));
          }
        }
        if (r < valid) {
#pragma unroll
          for (int i = 0; i < 32; i += 4)
            st_peer(dst + (c + i) * 4, __uint_as_float(v[i]), __uint_as_float(v[i + 1]), __uint_as_float(v[i + 2]), __uint_as_float(v[i + 3]));
        }
      }
    }
  }
  ptx::tc_fence_before_sync();
  __syncwarp();
  if (SPLITS > 1) { cluster_arrive(); cluster_wait(); }
  else __syncthreads();
  if (warp == 1) {
    ptx::tc_fence_after_sync();
    ptx::tmem_dealloc(tmem, kAccs * BN);
  }
  if (failed || !in) return;
  constexpr int kStep = kMidThreads / kQuads, U = 4;   // rows between a thread's, rows in flight
  const int own = min(share, valid - rank * share);
  const long long top = (long long)(row0 + rank * share) * p.cols + col;
  for (int first = tid / kQuads; first < own; first += U * kStep) {
    float4 s[U];
    Pack<TY, 4> res[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = first + u * kStep;
      if (p.lin.residual && r < own) res[u].load(static_cast<const TY*>(p.lin.residual) + top + (long long)r * p.cols);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float* at = sums + min(first + u * kStep, own - 1) * kLd + tid % kQuads * 4;
      s[u] = *reinterpret_cast<const float4*>(at);
#pragma unroll
      for (int k = 1; k < SPLITS; ++k) {
        const float4 v = *reinterpret_cast<const float4*>(at + k * share * kLd);
        s[u].x += v.x; s[u].y += v.y; s[u].z += v.z; s[u].w += v.w;
      }
      s[u].x += bias.x; s[u].y += bias.y; s[u].z += bias.z; s[u].w += bias.w;
    }
    if (p.lin.pre) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int r = first + u * kStep;
        const float f[4] = {s[u].x, s[u].y, s[u].z, s[u].w};
        if (r < own) store_pack<TY, 4>(static_cast<TY*>(p.lin.pre) + top + (long long)r * p.cols, f);
      }
    }
    uint32_t v[4 * U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      v[4 * u] = __float_as_uint(s[u].x); v[4 * u + 1] = __float_as_uint(s[u].y);
      v[4 * u + 2] = __float_as_uint(s[u].z); v[4 * u + 3] = __float_as_uint(s[u].w);
    }
    activate<4 * U, sizeof(TY) == 2>(v, p.lin.act);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = first + u * kStep;
      float f[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        f[j] = __uint_as_float(v[4 * u + j]);
        if (p.lin.residual) f[j] += res[u].get(j);
      }
      if (r < own) store_pack<TY, 4>(static_cast<TY*>(p.y) + top + (long long)r * p.cols, f);
    }
  }
}

template <bool A_K, bool B_K, int BN, int SPLITS, typename TY>
int launch_mid_t(const CUtensorMap& ma, const CUtensorMap& mb, const MidArgs& p_in, cudaStream_t st) {
  auto kern = linear_mid_kernel<A_K, B_K, BN, SPLITS, TY>;
  MidArgs p = p_in;
  const int stage = 2 * p.a_half + BN * kMidDepth * 2;
  const int valid = std::min(kMidRows, p.rows);
  const int sums = (valid + SPLITS - 1) / SPLITS * SPLITS * (BN + 4) * 4;
  const int room = kMidSmem - 1024 /*alignment*/ - kMidBarBytes - (SPLITS > 1 ? sums : 0);
  p.stages = std::min({kMidMaxStages, room / stage, std::max(2, p.run * p.passes)});
  // At least kMidAlone, which keeps any other kernel that allocates tensor memory off the multiprocessor: CTAs of two
  // clusters that waited for each other's tensor memory would never meet at their barriers.
  const int smem = std::max(kMidAlone, 1024 + kMidBarBytes + (SPLITS > 1 ? p.stages * stage + sums : std::max(p.stages * stage, sums)));
  // the same limit from every call: another thread may be between its own call of this and its launch
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kMidSmem) != cudaSuccess) {
    cudaGetLastError();
    return GSHARD_ERR_CUDA;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(SPLITS, ceil_div(p.cols, BN), ceil_div(p.rows, kMidRows));
  cfg.blockDim = dim3(kMidThreads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = SPLITS;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = SPLITS > 1 ? 1 : 0;
  if (cudaLaunchKernelEx(&cfg, kern, ma, mb, p) != cudaSuccess) { cudaGetLastError(); return GSHARD_ERR_CUDA; }
  count_launch();
  return GSHARD_OK;
}

template <bool A_K, bool B_K>
int launch_mid(const CUtensorMap& ma, const CUtensorMap& mb, const MidArgs& p, MidShape s, bool out_f32, cudaStream_t st) {
#define GSHARD_MID(S)                                                                      \
  case S:                                                                                  \
    if (out_f32) return launch_mid_t<A_K, B_K, 64, S, float>(ma, mb, p, st);               \
    return s.bn == 64 ? launch_mid_t<A_K, B_K, 64, S, __nv_bfloat16>(ma, mb, p, st)        \
                      : launch_mid_t<A_K, B_K, 128, S, __nv_bfloat16>(ma, mb, p, st);
  switch (s.splits) {
    GSHARD_MID(1)
    GSHARD_MID(2)
    GSHARD_MID(4)
  }
#undef GSHARD_MID
  return GSHARD_ERR_INTERNAL;
}

}  // namespace

// Measured against the general path (pairs of CTAs, tiles of 256 columns, runs joined by a second kernel), us: 64 rows of
// 1024 -> 1024 5.4 to 12.9, 8192 -> 1024 10.3 to 20.5, 4096 -> 4096 11.1 to 18.7; 512 rows of 1024 -> 1024 7.0 to 14.5,
// 4096 -> 4096 21.5 to 26.9.  Equal at 64 k-blocks per CTA (1024 rows of 8192 -> 1024: 26.0 to 26.8), and
// worse beyond.  Eight CTAs per cluster are no gain: 16 such clusters do not run at once (8192 -> 1024: 13 to 18), nor are
// more than 128 CTAs in clusters certain to.
MidShape linear_mid_shape(long long rows, int cols, long long depth, int passes, bool out_f32) {
  MidShape s{0, 1};
  const long long m_tiles = (rows + kMidRows - 1) / kMidRows, k_blocks = (depth + kMidDepth - 1) / kMidDepth;
  for (int bn = 64; bn <= (out_f32 ? 64 : 128) && !s.bn; bn *= 2)
    if (m_tiles * ceil_div(cols, bn) <= kMidSms) s.bn = bn;
  if (!s.bn) return s;
  const long long tiles = m_tiles * ceil_div(cols, s.bn);
  while (s.splits < 4 && 2 * s.splits * tiles <= 128 && k_blocks >= 4 * s.splits) s.splits *= 2;
  // no empty run at the end
  while (s.splits > 1 && (s.splits - 1) * ((k_blocks + s.splits - 1) / s.splits) >= k_blocks) s.splits /= 2;
  if ((k_blocks + s.splits - 1) / s.splits > most_k_blocks(passes, out_f32)) s.bn = 0;
  return s;
}

int launch_linear_mid(const UmmaGemm& g, const LinearEpilogue& lin, MidShape s, bool clear_status, int* status, cudaStream_t st) {
  if (g.batch != 1 || g.c_ld != g.cols || (!g.a_kmajor && g.b_kmajor)) return GSHARD_ERR_INTERNAL;
  const int pa = std::max(1, g.planes_a), pb = std::max(1, g.planes_b);
  const bool planes3 = pa == 3;
  if (planes3 ? pb != 3 || !g.out_f32 : pa * pb > 2 || (pa * pb == 2 && g.out_f32)) return GSHARD_ERR_INTERNAL;
  // Rows of A that are loaded: whole swizzle atoms of 8.  The MMA reads 128; what it finds behind the loaded ones goes
  // to accumulator rows that no one reads.
  const int a_rows = g.a_kmajor ? std::min(kMidRows, (g.rows + 7) / 8 * 8) : kMidRows;
  CUtensorMap ma, mb;
  bool ok = g.a_kmajor ? make_map(&ma, g.A, g.K, g.rows, pa, g.a_ld, g.a_bs, 64, a_rows)
                       : make_map(&ma, g.A, g.rows, g.K, pa, g.a_ld, g.a_bs, 64, kMidDepth);
  ok = ok && (g.b_kmajor ? make_map(&mb, g.B, g.K, g.cols, pb, g.b_ld, g.b_bs, 64, s.bn)
                         : make_map(&mb, g.B, g.cols, g.K, pb, g.b_ld, g.b_bs, 64, kMidDepth));
  if (!ok) return GSHARD_ERR_CUDA;
  MidArgs p{};
  p.y = g.C; p.lin = lin; p.status = status; p.clear_status = clear_status; p.rows = g.rows; p.cols = g.cols;
  p.k_blocks = ceil_div(g.K, kMidDepth);
  p.run = ceil_div(p.k_blocks, s.splits);
  p.passes = planes3 ? umma_epi::kPasses3 : pa * pb;
  p.pass_a = planes3 ? umma_epi::kPassA3 : pa == 2 ? 0x01 : 0;     // two planes: the low one first
  p.pass_b = planes3 ? umma_epi::kPassB3 : pb == 2 ? 0x01 : 0;
  p.a_half = a_rows * 128;
  p.a_once = g.cols <= s.bn;
  p.b_once = g.rows <= kMidRows;
  const bool out_f32 = g.out_f32 != 0;
  if (!g.a_kmajor) return launch_mid<false, false>(ma, mb, p, s, out_f32, st);
  return g.b_kmajor ? launch_mid<true, true>(ma, mb, p, s, out_f32, st) : launch_mid<true, false>(ma, mb, p, s, out_f32, st);
}

}  // namespace gshard
