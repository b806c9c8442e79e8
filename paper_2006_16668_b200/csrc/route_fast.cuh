// Routing kernels that hold a token's logits in registers: LPR lanes of a warp (8 or 32) share a token, V
// logits each, and the other lanes work on further tokens.  Included by one source file per logits type.
//
// What bounds the pass: the logits are read once, so HBM while few experts are chosen, the arithmetic of
// the choice with many.  Measured: 131072 tokens, top-2 of 2048 fp32 190 us (5.7 TB/s), with mean gates 264; 65536
// tokens, sigmoid + bias, 4 of 8 groups, top-8 of 512 bf16 97 us, of which the nine picks 29, the groups 16.  Reductions and
// the bookkeeping of a pick cost about the same however many tokens the warp holds, which is why eight
// lanes per token are taken where the experts fit.
// Layout: lanes take turns of W consecutive experts, so that loads are whole 16-byte words (W = 1 for rows that are
// not).  The values that decide the choice lie in shared memory, in chunks of 8 per lane with the chunk's maximum in a
// register: a pick then looks at one chunk of one lane instead of at all its values.  With groups LPR / groups
// lanes own a group, and the values change lanes on their way through shared memory (loading each group by
// its owners costs four times the L1 passes).
#pragma once
#include "route.cuh"

namespace gshard {

namespace {

constexpr int kRouteThreads = 128;
constexpr int kRouteWarps = kRouteThreads / 32;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// 1 / (1 + exp(-l)) to about 2^-22: two approximate operations of 1 to 2 units in the last place
__device__ __forceinline__ float sigmoid_fast(float l) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(1.f + exp2_approx(-l * kLog2e)));
  return y;
}

// exp(l - mx), up to a factor close to 1 that is the same for the whole row: below 2^20 the shift -mx log2(e) is rounded
// before the logits' products with log2(e) are added to it exactly.  So a sum of these may be divided into these only: the
// factor is 2^(half a step of the shift), 5e-6 at logits near 100 and 4 % near 10^6.
__device__ __forceinline__ float row_exp(float l, float mx) {
  return exp2_approx(fabsf(mx) <= 0x1p20f ? fmaf(l, kLog2e, -mx * kLog2e) : (l - mx) * kLog2e);
}

// s (1 - s) of s = sigmoid(l): with e = exp(-|l|) it is e / (1 + e)^2, which loses nothing where s is close to 1 (s times
// the difference 1 - s is 0.2 % off at l = 10 and 0 from 17 on)
__device__ __forceinline__ float sigmoid_slope_fast(float l) {
  const float e = exp2_approx(-fabsf(l) * kLog2e);
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
  return e * r * r;
}

template <int LPR> __device__ __forceinline__ float seg_max(float v) {
#pragma unroll
  for (int off = LPR / 2; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor_sync(kAll, v, off));
  return v;
}
template <int LPR> __device__ __forceinline__ float seg_sum(float v) {
#pragma unroll
  for (int off = LPR / 2; off > 0; off >>= 1) v += __shfl_xor_sync(kAll, v, off);
  return v;
}
template <int LPR> __device__ __forceinline__ int seg_min(int v) {
#pragma unroll
  for (int off = LPR / 2; off > 0; off >>= 1) v = min(v, __shfl_xor_sync(kAll, v, off));
  return v;
}
// chosen_ratio for a token held by LPR lanes
template <int LPR> __device__ __forceinline__ float seg_ratio(float l, int sigmoid, float& total) {
  float top = seg_max<LPR>(l);
  if (top == -INFINITY) top = 0.f;
  float r;
  if (!sigmoid) r = expf(l - top);
  else if (top < 0.f) r = expf(l - top) * (1.f + expf(top)) / (1.f + expf(fminf(l, 0.f)));
  else r = (1.f + expf(-top)) / (1.f + expf(-l));
  if (l == -INFINITY) r = 0.f;
  total = seg_sum<LPR>(r);
  return r;
}

// Where a lane's values lie in the row.
template <int W> struct RouteLane {
  int base, q, P, size;     // first expert of the lane's group, lane inside the group, lanes per group, experts per group
  __device__ __forceinline__ int offset(int i) const { return ((i / W) * P + q) * W + i % W; }   // inside the group
  __device__ __forceinline__ int expert(int i) const { return base + offset(i); }
};

// V logits of this lane; -inf beyond the group's end (`full`: the group fills the lanes exactly).
template <typename T, int W, int V>
__device__ __forceinline__ void load_logits(const T* row, const RouteLane<W>& ln, bool full, float (&v)[V]) {
  if (full) {
#pragma unroll
    for (int j = 0; j < V / W; ++j) load_pack<T, W>(row + ln.base + (j * ln.P + ln.q) * W, v + j * W);
  } else {
#pragma unroll
    for (int j = 0; j < V / W; ++j) {
      const int off = (j * ln.P + ln.q) * W;
      if (off < ln.size) {
        load_pack<T, W>(row + ln.base + off, v + j * W);
      } else {
#pragma unroll
        for (int w = 0; w < W; ++w) v[j * W + w] = -INFINITY;
      }
    }
  }
}
// NaN bars like -inf, +inf counts as the largest float
template <int V> __device__ __forceinline__ void clean(float (&v)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = fminf(fmaxf(v[i], -INFINITY), FLT_MAX);
}

// Shared memory of a warp: V / 4 units of 32 x 16 bytes; a lane's values i .. i + 3 (i a multiple of 4) are unit i / 4.
// The lane is XORed with the unit (per vector of W), which spreads the stores of values that change lanes over the banks.
template <int W> __device__ __forceinline__ int unit_at(int unit, int lane) {
  return (unit * 32 + (lane ^ ((W >= 4 ? unit / (W / 4) : unit) & 7))) * 4;
}
template <int W> __device__ __forceinline__ void chunk_values(const float* st, int lane, int c, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; i += 4) {
    const float4 f = *reinterpret_cast<const float4*>(st + unit_at<W>(c * 2 + i / 4, lane));
    x[i] = f.x; x[i + 1] = f.y; x[i + 2] = f.z; x[i + 3] = f.w;
  }
}

// A score in 64 bits; norm: the 64-bit sum of exp(l - mx) over the row (softmax).
__device__ __noinline__ double score64(float l, int sigmoid, float mx, double norm) {
  return sigmoid ? 1.0 / (1.0 + exp(-(double)l)) : exp((double)l - (double)mx) / norm;
}
template <int LPR, int V, int W, typename T>
__device__ __noinline__ double softmax_norm64(const T* row, const RouteLane<W>& ln, float mx) {
  double s = 0.0;
#pragma unroll 1
  for (int i = 0; i < V; ++i)
    if (ln.offset(i) < ln.size) s += exp((double)usable(row[ln.expert(i)]) - (double)mx);
#pragma unroll
  for (int off = LPR / 2; off > 0; off >>= 1) s += __shfl_xor_sync(kAll, s, off);
  return s > 0.0 ? s : 1.0;
}

// What decides the choice: the logits; a softmax's scores plus bias; logits, with groups valued by sums of scores; or a
// sigmoid's scores plus bias, which need no sum over the row, so that its logits pass through the registers in pieces.
enum RouteMode { kByLogits = 0, kBySoftmaxBias = 1, kBySums = 2, kBySigmoidBias = 3 };

// MEAN: sums of the scores over the block's tokens, in registers, or (64 values per lane) in shared memory, where
// they leave the registers to more warps.
template <typename T, int W, int LPR, int V, int MODE, bool MEAN>
__global__ void __launch_bounds__(kRouteThreads, V < 64 || W == 1 ? 1 : MODE == kBySigmoidBias ? (MEAN ? 3 : 4) : MEAN && MODE == kByLogits ? 3 : 4)
route_fwd_fast_kernel(const __grid_constant__ RouteArgs a, float* __restrict__ sums) {
  constexpr int RPW = 32 / LPR;               // tokens per warp
  constexpr int NC = V / 8;
  constexpr bool ACC_SMEM = MEAN && V == 64, BIASED = MODE != kByLogits, STREAM = MODE == kBySigmoidBias;
  constexpr bool by_bias = MODE == kBySoftmaxBias || STREAM;
  extern __shared__ __align__(16) float route_smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int slot = lane / LPR, p = lane % LPR;
  float* st = route_smem + warp * V * 32;                       // the values that decide; at the end the sums
  float* sacc = route_smem + (warp + kRouteWarps) * V * 32;     // ACC_SMEM
  const RouteLane<W> lin{0, p, LPR, a.E};     // as loaded
  RouteLane<W> ln;                            // as owned for the choice: the same without groups
  ln.P = LPR / a.groups; ln.q = p % ln.P; ln.size = a.E / a.groups; ln.base = p / ln.P * ln.size;
  const bool grouped = a.groups > 1;
  const bool full = a.E == V * LPR, owns_all = ln.size == V * ln.P;
  const bool need_sum = !STREAM && !a.sigmoid && (MEAN || !a.renorm || BIASED);
  const int t0 = blockIdx.x * kRouteTile, t1 = min(a.S, t0 + kRouteTile);
  const long long first = (long long)blockIdx.y * a.S;
  // group of vector vi: vi / per_group by a 32-bit reciprocal (exact while vi * per_group < 2^32; 1 divides nothing)
  const unsigned per_group = ln.size / W, recip = 0xffffffffu / per_group + 1u;
  const int lg = __ffs(ln.P) - 1;
  // a vector of this lane to where its owner looks for it
  auto stage = [&](int j, const float* x, bool moves) {
    int unit = j * W / 4, to = lane, comp = j * W % 4;
    if (moves) {
      const int vi = j * LPR + p, g = per_group == 1 ? vi : (int)__umulhi((unsigned)vi, recip), r = vi - g * (int)per_group;
      to = slot * LPR + (g << lg) + (r & (ln.P - 1));
      const int i = (r >> lg) * W;
      unit = i / 4; comp = i % 4;
      if (vi * W >= a.E) return;
    }
    if constexpr (W >= 4) {
#pragma unroll
      for (int w = 0; w < W; w += 4)
        *reinterpret_cast<float4*>(st + unit_at<W>(unit + w / 4, to)) = make_float4(x[w], x[w + 1], x[w + 2], x[w + 3]);
    } else {
      st[unit_at<W>(unit, to) + comp] = x[0];
    }
  };
  auto blank = [&]() {                        // places beyond a group's end: nothing is ever staged there
    if (grouped && !owns_all) {
#pragma unroll
      for (int u = 0; u < V / 4; ++u) *reinterpret_cast<float4*>(st + unit_at<W>(u, lane)) = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
    }
  };
  blank();
  float acc[MEAN && !ACC_SMEM ? V : 4];
  if (MEAN && !ACC_SMEM) {
#pragma unroll
    for (int i = 0; i < V; ++i) acc[ACC_SMEM ? 0 : i] = 0.f;
  }
  if (ACC_SMEM) {
#pragma unroll
    for (int i = 0; i < V; i += 4) *reinterpret_cast<float4*>(sacc + (i / 4 * 32 + lane) * 4) = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  // f * s[0..4) of an active token to the sums i .. i + 3
  auto accumulate = [&](int i, const float* s, float f) {
    const f32x2 ff = both(f);
    if (ACC_SMEM) {
      float4* at = reinterpret_cast<float4*>(sacc + (i / 4 * 32 + lane) * 4);
      const float4 o = *at;
      const float2 lo = unpair(fma2(pair(s[0], s[1]), ff, pair(o.x, o.y)));
      const float2 hi = unpair(fma2(pair(s[2], s[3]), ff, pair(o.z, o.w)));
      *at = make_float4(lo.x, lo.y, hi.x, hi.y);
    } else {
#pragma unroll
      for (int w = 0; w < 4; w += 2) {
        const float2 o = unpair(fma2(pair(s[w], s[w + 1]), ff, pair(acc[ACC_SMEM ? 0 : i + w], acc[ACC_SMEM ? 1 : i + w + 1])));
        acc[ACC_SMEM ? 0 : i + w] = o.x; acc[ACC_SMEM ? 1 : i + w + 1] = o.y;
      }
    }
  };

  for (int s0 = t0 + warp * RPW; s0 < t1; s0 += kRouteWarps * RPW) {
    const bool active = s0 + slot < t1;
    const long long t = first + min(s0 + slot, t1 - 1);
    const T* row = static_cast<const T*>(a.logits) + t * a.E;
    float v[STREAM ? W : V];
    if constexpr (!STREAM) load_logits<T, W, V>(row, lin, full, v);
    {                                          // the warp's next tokens on their way into L2 meanwhile
      const int s1 = s0 + kRouteWarps * RPW;
      const char* ahead = reinterpret_cast<const char*>(static_cast<const T*>(a.logits) + (first + s1) * a.E);
      const int bytes = min(RPW, t1 - s1) * a.E * (int)sizeof(T);
      for (int o = lane * 128; o < bytes; o += 4096) asm volatile("prefetch.global.L2 [%0];" ::"l"(ahead + o));
    }
    float cm[NC];
    float mx = -INFINITY, inv = 0.f;
    double norm64 = 0.0;                       // 64-bit sum of a softmax, once something needs it
    // Errors of fp32 scores: of a softmax, (V + 32) roundings of its sum and its exponentials; of a sigmoid,
    // under 2^-20; the sum with the bias half a step.  Values closer than twice that are compared in 64 bits.
    float slack = 0x1p-20f;
    __syncwarp();                              // the previous tokens' values have been read
    if constexpr (MODE == kBySums) clean<V>(v);
    if constexpr (!by_bias) {
      auto maxima = [&]() {
        mx = -INFINITY;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          float m = v[c * 8];
#pragma unroll
          for (int i = 1; i < 8; ++i) m = fmaxf(m, v[c * 8 + i]);
          cm[c] = fmaxf(m, -INFINITY);
          mx = fmaxf(mx, cm[c]);
        }
      };
      maxima();
      // fmaxf passes over NaN, so that logits need no clean-up for the choice, except that +inf and the largest float
      // are the same
      if (MODE == kByLogits && __any_sync(kAll, mx == INFINITY)) { clean<V>(v); maxima(); }
      if (grouped) {
#pragma unroll
        for (int j = 0; j < V / W; ++j) stage(j, v + j * W, true);
      } else {
#pragma unroll
        for (int j = 0; j < V / W; ++j) stage(j, v + j * W, false);
      }
    }
    if constexpr (MODE == kByLogits) {
      // exponentials of NaN or of infinite logits are caught by the two tests below
      if (need_sum) {
        mx = seg_max<LPR>(mx);
        const float shift = -mx * kLog2e;      // row_exp of all values, two at a time
        f32x2 sum2x[2] = {both(0.f), both(0.f)};
#pragma unroll
        for (int i = 0; i < V; i += 2) {
          const float2 e = unpair(fma2(pair(v[i], v[i + 1]), both(kLog2e), both(shift)));
          v[i] = exp2_approx(e.x); v[i + 1] = exp2_approx(e.y);
          sum2x[i / 2 % 2] = add2(sum2x[i / 2 % 2], pair(v[i], v[i + 1]));
        }
        const float2 sums2 = unpair(add2(sum2x[0], sum2x[1]));
        float sum = seg_sum<LPR>(sums2.x + sums2.y);
        const bool odd = !(fabsf(mx) <= 0x1p20f) || !(sum < INFINITY);
        if (__any_sync(kAll, odd)) {           // NaN, infinite or huge logits, or no expert at all: once more, cleaned up
          float m2 = -INFINITY, sum2 = 0.f;
#pragma unroll 1
          for (int i = 0; i < V; ++i)
            if (lin.offset(i) < a.E) m2 = fmaxf(m2, usable(row[lin.expert(i)]));
          m2 = seg_max<LPR>(m2);
          if (m2 == -INFINITY) m2 = 0.f;
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const float l = lin.offset(i) < a.E ? usable(row[lin.expert(i)]) : -INFINITY;
            const float e = row_exp(l, m2);
            sum2 += e;
            if (odd) v[i] = e;
          }
          sum2 = seg_sum<LPR>(sum2);
          if (odd) { mx = m2; sum = sum2; }
        }
        inv = sum > 0.f ? 1.f / sum : 0.f;
      }
      if (MEAN && a.sigmoid) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = sigmoid_fast(fmaxf(v[i], -INFINITY));
      }
      if (MEAN && active) {
#pragma unroll
        for (int i = 0; i < V; i += 4) accumulate(i, v + i, a.sigmoid ? 1.f : inv);
      }
    } else if constexpr (STREAM) {
      constexpr int Q = V / W < 4 ? V / W : 4;               // vectors on their way at a time
#pragma unroll
      for (int jb = 0; jb < V / W; jb += Q) {
        Pack<T, W> q[Q];
#pragma unroll
        for (int u = 0; u < Q; ++u) {
          const int off = ((jb + u) * LPR + p) * W;
          if (full || off < a.E) q[u].load(row + off);
        }
#pragma unroll
        for (int u = 0; u < Q; ++u) {
          constexpr int C = W < 4 ? W : 4;
          const int j = jb + u, off = (j * LPR + p) * W;
          float b[W], s[W], x[W];
          if (full || off < a.E) {
#pragma unroll
            for (int w = 0; w < W; w += C) load_pack<float, C>(a.bias + off + w, b + w);
#pragma unroll
            for (int w = 0; w < W; ++w) {
              const float l = q[u].get(w);
              s[w] = sigmoid_fast(l);                        // NaN logits and biases: barred by the maximum
              x[w] = l == -INFINITY ? -INFINITY : fmaxf(s[w] + b[w], -INFINITY);
            }
          } else {
#pragma unroll
            for (int w = 0; w < W; ++w) { s[w] = 0.f; x[w] = -INFINITY; }
          }
          stage(j, x, grouped);
          if constexpr (MEAN) {
            static_assert(!MEAN || W >= 4 || W == 1, "");
#pragma unroll
            for (int w = 0; w < W; ++w) s[w] = active ? fmaxf(s[w], 0.f) : 0.f;
            if constexpr (W >= 4) {
#pragma unroll
              for (int w = 0; w < W; w += 4) accumulate(j * W + w, s + w, 1.f);
            } else {
              float one[4] = {0.f, 0.f, 0.f, 0.f};
              one[j % 4] = s[0];
              accumulate(j / 4 * 4, one, 1.f);
            }
          }
          if (!grouped) {
#pragma unroll
            for (int w = 0; w < W; ++w) cm[(j * W + w) / 8] = (j * W + w) % 8 == 0 ? x[w] : fmaxf(cm[(j * W + w) / 8], x[w]);
          }
        }
      }
    } else {
      if (need_sum) {
        if (by_bias) clean<V>(v);
        mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < V; ++i) mx = fmaxf(mx, v[i]);
        mx = seg_max<LPR>(mx);
        if (mx == -INFINITY) mx = 0.f;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) sum += exp2_approx((v[i] - mx) * kLog2e);
        sum = seg_sum<LPR>(sum);
        inv = sum > 0.f ? 1.f / sum : 0.f;
        slack = (V + 32) * 0x1p-24f * inv;
      }
      if (by_bias || MEAN) {
        // scores into v; then the values that decide
#pragma unroll
        for (int j = 0; j < V / W; ++j) {
          float s[W], x[W];
          if (MODE == kBySums && a.sigmoid) {
#pragma unroll
            for (int w = 0; w < W; ++w) s[w] = sigmoid_fast(v[j * W + w]);
          } else {
#pragma unroll
            for (int w = 0; w < W; ++w) s[w] = exp2_approx((v[j * W + w] - mx) * kLog2e) * inv;
          }
          if (by_bias) {
            constexpr int C = W < 4 ? W : 4;
            float b[W];
            const int off = (j * LPR + p) * W;
#pragma unroll
            for (int w = 0; w < W; ++w) b[w] = 0.f;
            if (full || off < a.E) {
#pragma unroll
              for (int w = 0; w < W; w += C) load_pack<float, C>(a.bias + off + w, b + w);
            }
#pragma unroll
            for (int w = 0; w < W; ++w) x[w] = v[j * W + w] == -INFINITY ? -INFINITY : fmaxf(s[w] + b[w], -INFINITY);
            stage(j, x, grouped);
          }
#pragma unroll
          for (int w = 0; w < W; ++w) v[j * W + w] = MEAN ? s[w] : x[w];
        }
        if (MEAN && active) {
#pragma unroll
          for (int i = 0; i < V; i += 4) accumulate(i, v + i, 1.f);
        }
      }
    }
    if (grouped || (MEAN && MODE == kBySoftmaxBias)) {        // maxima of the chunks as they are owned
      __syncwarp();
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        float x[8];
        chunk_values<W>(st, lane, c, x);
        cm[c] = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8; ++i) cm[c] = fmaxf(cm[c], x[i]);
      }
    } else if constexpr (MODE == kBySoftmaxBias) {
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        cm[c] = v[c * 8];
#pragma unroll
        for (int i = 1; i < 8; ++i) cm[c] = fmaxf(cm[c], v[c * 8 + i]);
      }
    }
    if (grouped) {
      float top1 = -INFINITY, top2 = -INFINITY;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        top2 = fmaxf(top2, fminf(top1, cm[c]));
        top1 = fmaxf(top1, cm[c]);
      }
      if (BIASED && a.group_top == 2) {        // the runner-up may share the best one's chunk
        int bc = 0;
#pragma unroll
        for (int c = NC - 1; c >= 0; --c)
          if (cm[c] == top1) bc = c;
        float x[8], x1 = -INFINITY, x2 = -INFINITY;
        chunk_values<W>(st, lane, bc, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) { x2 = fmaxf(x2, fminf(x1, x[i])); x1 = fmaxf(x1, x[i]); }
        top2 = fmaxf(top2, x2);
      }
      for (int off = 1; off < ln.P; off <<= 1) {
        const float o1 = __shfl_xor_sync(kAll, top1, off), o2 = __shfl_xor_sync(kAll, top2, off);
        top2 = fmaxf(fminf(top1, o1), fmaxf(top2, o2));
        top1 = fmaxf(top1, o1);
      }
      const float floor2 = a.group_top == 2 ? top2 : top1;
      if (MODE == kBySums) {                   // logits so far: scores grow with them
        top1 = top1 == -INFINITY ? top1 : a.sigmoid ? sigmoid_fast(top1) : exp2_approx((fminf(top1, FLT_MAX) - mx) * kLog2e) * inv;
        top2 = top2 == -INFINITY ? top2 : a.sigmoid ? sigmoid_fast(top2) : exp2_approx((fminf(top2, FLT_MAX) - mx) * kLog2e) * inv;
      }
      const float mine = BIASED && a.group_top == 2 && top2 != -INFINITY ? top1 + top2 : top1;
      const int group = p >> lg;
      int better = 0;
      for (int g = 0; g < a.groups; ++g) {
        const float other = __shfl_sync(kAll, mine, slot * LPR + (g << lg));
        better += (other > mine || (other == mine && g < group)) ? 1 : 0;
      }
      bool keep = better < a.kept;
      if (BIASED) {
        // What this group's value may be off by: its entries' scores, and half a step of each entry and of their sum, which
        // may be far smaller than either (a score plus a large bias and a score minus it).
        const float second = a.group_top == 2 && top2 != -INFINITY ? top2 : 0.f;
        const float off = 2.f * slack + 0x1p-21f * fmaxf(top1 == -INFINITY ? 0.f : fabsf(top1), fabsf(second));
        const float worst_kept = -seg_max<LPR>(keep ? off - mine : -INFINITY);
        const float best_left = seg_max<LPR>(keep ? -INFINITY : mine + off);
        const bool near = best_left != -INFINITY && worst_kept <= best_left;
        if (__any_sync(kAll, near)) {
          // the groups' values again in 64 bits, from the few entries that can be among a group's best
          if (!a.sigmoid && norm64 == 0.0) norm64 = softmax_norm64<LPR, V>(row, lin, mx);
          const float from = floor2 - (by_bias ? 2.f * slack + 0x1p-21f * fabsf(floor2) : 0.f);
          double d1 = -INFINITY, d2 = -INFINITY;
#pragma unroll 1
          for (int c = 0; c < NC; ++c) {
            float x[8];
            chunk_values<W>(st, lane, c, x);
            for (int i = 0; i < 8; ++i) {
              if (!(x[i] > -INFINITY) || !(x[i] >= from || floor2 == -INFINITY)) continue;
              const int e = ln.expert(c * 8 + i);
              const double d = score64(usable(row[e]), a.sigmoid, mx, norm64) + (by_bias ? (double)a.bias[e] : 0.0);
              if (d > d1) { d2 = d1; d1 = d; } else if (d > d2) d2 = d;
            }
          }
          for (int off = 1; off < ln.P; off <<= 1) {
            const double o1 = __shfl_xor_sync(kAll, d1, off), o2 = __shfl_xor_sync(kAll, d2, off);
            d2 = fmax(fmin(d1, o1), fmax(d2, o2));
            d1 = fmax(d1, o1);
          }
          const double mine64 = a.group_top == 2 && d2 != -INFINITY ? d1 + d2 : d1;
          better = 0;
          for (int g = 0; g < a.groups; ++g) {
            const double other = __shfl_sync(kAll, mine64, slot * LPR + (g << lg));
            better += (other > mine64 || (other == mine64 && g < group)) ? 1 : 0;
          }
          keep = better < a.kept;
        }
      }
      if (!keep) {
#pragma unroll
        for (int c = 0; c < NC; ++c) cm[c] = -INFINITY;
      }
    }
    // Picks.  The lanes whose best value is the token's best look up which one it is (the lowest index wins); the
    // winner blots it out and takes its chunk's maximum again.
    // With a bias fp32 values that are too close to call are looked at again: the picks go on behind the k-th as
    // long as its value is not clearly larger, and lane p also holds the (p + LPR)-th of them.
    float bv = cm[0];
#pragma unroll
    for (int c = 1; c < NC; ++c) bv = fmaxf(bv, cm[c]);
    int picked = -1, extra = -1, held = a.k;
    float value = -INFINITY, before = INFINITY, kth = INFINITY;
    bool near = false, more = by_bias;
    for (int j = 0; j < a.k || (by_bias && j < 2 * LPR && __any_sync(kAll, more)); ++j) {
      const float gv = seg_max<LPR>(bv);
      int e = INT_MAX, bi = 0, bc = 0;
      const bool mine = bv == gv && gv != -INFINITY;
      if (mine) {
#pragma unroll
        for (int c = NC - 1; c >= 0; --c)
          if (cm[c] == bv) bc = c;
        float x[8];
        chunk_values<W>(st, lane, bc, x);
#pragma unroll
        for (int i = 7; i >= 0; --i)
          if (x[i] == bv) bi = i;
        bi += bc * 8;
        e = ln.expert(bi);
      }
      const int ge = seg_min<LPR>(e);
      if (by_bias) {
        const float top = j < a.k ? before : kth;
        const bool tight = gv != -INFINITY && top - gv <= 2.f * slack + 0x1p-22f * fmaxf(fabsf(top), fabsf(gv));
        if (j >= a.k) {
          more = more && tight;
          if (more) { held = j + 1; near = true; }
        } else if (j > 0 && tight) {
          near = true;
        }
        before = gv;
        if (j == a.k - 1) kth = gv;
      }
      const int got = ge == INT_MAX || (by_bias && j >= a.k && !more) ? -1 : ge;
      if (p == j) { picked = got; value = gv; }
      if (by_bias && p + LPR == j) extra = got;
      if (mine && e == ge) {
        st[unit_at<W>(bi / 4, lane) + bi % 4] = -INFINITY;
        float x[8], left = -INFINITY;
        chunk_values<W>(st, lane, bc, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) left = fmaxf(left, x[i]);
        bv = -INFINITY;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          if (c == bc) cm[c] = left;
          bv = fmaxf(bv, cm[c]);
        }
      }
    }
    if (by_bias && __any_sync(kAll, near)) {
      if (!a.sigmoid && norm64 == 0.0) norm64 = softmax_norm64<LPR, V>(row, lin, mx);
      // held picks by their 64-bit values; lane p's two are picks p and p + LPR
      auto value64 = [&](int e) -> double {
        return e < 0 ? -INFINITY : score64(usable(row[e]), a.sigmoid, mx, norm64) + (double)a.bias[e];
      };
      const double c0 = value64(picked), c1 = extra >= 0 ? value64(extra) : -INFINITY;
      int rank0 = 0, rank1 = 0;
      const int most = __reduce_max_sync(kAll, held);
      for (int q = 0; q < most; ++q) {
        const int from = slot * LPR + q % LPR;
        const double oc0 = __shfl_sync(kAll, c0, from), oc1 = __shfl_sync(kAll, c1, from);
        const int oe0 = __shfl_sync(kAll, picked, from), oe1 = __shfl_sync(kAll, extra, from);
        const double oc = q < LPR ? oc0 : oc1;
        const int oe = q < LPR ? oe0 : oe1;
        if (oe >= 0 && (oc > c0 || (oc == c0 && oe < picked))) ++rank0;
        if (oe >= 0 && (oc > c1 || (oc == c1 && oe < extra))) ++rank1;
      }
      int sorted = -1;
      for (int q = 0; q < most; ++q) {
        const int from = slot * LPR + q % LPR;
        const int r0 = __shfl_sync(kAll, rank0, from), r1 = __shfl_sync(kAll, rank1, from);
        const int oe0 = __shfl_sync(kAll, picked, from), oe1 = __shfl_sync(kAll, extra, from);
        const int r = q < LPR ? r0 : r1, oe = q < LPR ? oe0 : oe1;
        if (oe >= 0 && r == p) sorted = oe;
      }
      if (near) picked = sorted;
      // more near ties than the lanes hold: the whole row in 64 bits
      unsigned open = __ballot_sync(kAll, more && active && p == 0);
      const bool reuse = open != 0;
      while (open) {
        const int src = __ffs(open) - 1;
        open &= open - 1;
        const long long tt = __shfl_sync(kAll, t, src);
        double* cache = a.E <= V * 16 ? reinterpret_cast<double*>(st) : nullptr;
        const int e = choose_exact<T>(static_cast<const T*>(a.logits) + tt * a.E, a, lane, cache);
        const int ep = __shfl_sync(kAll, e, p);
        if (slot == src / LPR) picked = p < a.k ? ep : -1;
      }
      if (reuse) blank();
    }
    if (p >= a.k) picked = -1;
    // without a bias the value that was compared is the logit
    const float l = picked < 0 ? -INFINITY : by_bias ? usable(row[picked]) : fminf(value, FLT_MAX);
    float w;
    if (a.renorm) {
      float total;
      w = seg_ratio<LPR>(l, a.sigmoid, total);
      w = total > 0.f ? a.scale * (w / total) : 0.f;
    } else {
      // by logits the sum was taken over row_exp, otherwise over exponentials of differences
      w = picked < 0 ? 0.f : a.scale * (a.sigmoid ? sigmoid_f(l) : (MODE == kByLogits ? row_exp(l, mx) : expf(l - mx)) * inv);
    }
    if (active && p < a.k) {
      a.expert_idx[t * a.k + p] = picked;
      a.weight[t * a.k + p] = w;
      if (a.load && picked >= 0) atomicAdd(a.load + (long long)blockIdx.y * a.E + picked, 1);
    }
  }

  if (MEAN) {                                  // the block's sum: warps in order, within each the tokens side by side
    if (!ACC_SMEM) {
      __syncwarp();
#pragma unroll
      for (int i = 0; i < V; i += 4)
        *reinterpret_cast<float4*>(st + (i / 4 * 32 + lane) * 4) =
            make_float4(acc[ACC_SMEM ? 0 : i], acc[ACC_SMEM ? 1 : i + 1], acc[ACC_SMEM ? 2 : i + 2], acc[ACC_SMEM ? 3 : i + 3]);
    }
    const float* all = route_smem + (ACC_SMEM ? kRouteWarps * V * 32 : 0);
    __syncthreads();
    const float scale = gridDim.x == 1 ? 1.f / (float)a.S : 1.f;       // a single tile is the mean already
    float* out = sums + ((long long)blockIdx.y * gridDim.x + blockIdx.x) * a.E;
    for (int c = threadIdx.x; c < V * LPR; c += kRouteThreads) {
      const int i = c / (LPR * 4) * 4 + c % 4, pp = c / 4 % LPR;
      const RouteLane<W> o{0, pp, LPR, a.E};
      if (o.offset(i) < a.E) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < kRouteWarps; ++w)
#pragma unroll
          for (int r = 0; r < RPW; ++r) s += all[w * V * 32 + (i / 4 * 32 + r * LPR + pp) * 4 + i % 4];
        out[o.expert(i)] = s * scale;
      }
    }
  }
}

// Gradient (see route_bwd_kernel for the formulas).
template <typename T, int W, int LPR, int V>
__global__ void __launch_bounds__(kRouteThreads) route_bwd_fast_kernel(const RouteGradArgs a) {
  constexpr int RPW = 32 / LPR;
  const int lane = threadIdx.x & 31;
  const int slot = lane / LPR, p = lane % LPR;
  const RouteLane<W> ln{0, p, LPR, a.E};
  const bool soft_stats = !a.sigmoid && (a.dm || !a.renorm);
  const bool dense = soft_stats || a.dm;
  const float inv_s = 1.f / (float)a.S;
  const long long step = (long long)gridDim.x * kRouteWarps * RPW;
  for (long long b0 = ((long long)blockIdx.x * kRouteWarps + (threadIdx.x >> 5)) * RPW; b0 < a.n; b0 += step) {
    const bool active = b0 + slot < a.n;
    const long long t = active ? b0 + slot : a.n - 1;
    const T* row = static_cast<const T*>(a.logits) + t * a.E;
    T* out = static_cast<T*>(a.dlogits) + t * a.E;
    const float* dm = a.dm ? a.dm + t / a.S * a.E : nullptr;
    float v[V];
    if (dense) load_logits<T, W, V>(row, ln, a.E == V * LPR, v);    // in flight while the picks' own loads follow one another
    int e = -1;
    float l = -INFINITY, dw = 0.f;
    if (p < a.k) {
      e = a.expert_idx[t * a.k + p];
      if (e < 0 || e >= a.E) e = -1;
      if (e >= 0) { l = usable(row[e]); dw = a.dweight[t * a.k + p]; }
      if (l == -INFINITY) e = -1;
    }
    float mx = 0.f, inv = 0.f;
    if (dense) {
      clean<V>(v);
      if (soft_stats) {
        mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < V; ++i) mx = fmaxf(mx, v[i]);
        mx = seg_max<LPR>(mx);
        if (mx == -INFINITY) mx = 0.f;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) { v[i] = exp2_approx((v[i] - mx) * kLog2e); sum += v[i]; }
        sum = seg_sum<LPR>(sum);
        inv = sum > 0.f ? 1.f / sum : 0.f;
      }
    }
    float add = 0.f;
    if (a.renorm) {
      float total;
      const float r = seg_ratio<LPR>(l, a.sigmoid, total);
      const float w = total > 0.f ? r / total : 0.f;
      const float D = seg_sum<LPR>(e >= 0 ? w * dw : 0.f);
      add = e >= 0 ? a.scale * w * (dw - D) : 0.f;
      if (a.sigmoid && e >= 0) add /= 1.f + expf(l);
    } else if (e >= 0) {
      const float s = a.sigmoid ? sigmoid_f(l) : expf(l - mx) * inv;
      add = a.scale * dw * s;
      if (a.sigmoid) add /= 1.f + expf(l);
    }
    float dot = 0.f;
    if (soft_stats) {
      if (dm) {
#pragma unroll
        for (int j = 0; j < V / W; ++j) {
          const int off = (j * LPR + p) * W;
          if (off < a.E) {
            constexpr int C = W < 4 ? W : 4;
            float d[W];
#pragma unroll
            for (int w = 0; w < W; w += C) load_pack<float, C>(dm + off + w, d + w);
#pragma unroll
            for (int w = 0; w < W; ++w) dot = fmaf(v[j * W + w], d[w], dot);
          }
        }
        dot *= inv * inv_s;
      }
      dot = seg_sum<LPR>(dot + (a.renorm ? 0.f : add));
    }
    float sum = add;
    bool writes = e >= 0;
    for (int j = 0; j < a.k; ++j) {              // entries that name the same expert add up; the first of them writes
      const int oe = __shfl_sync(kAll, e, slot * LPR + j);
      const float oa = __shfl_sync(kAll, add, slot * LPR + j);
      if (j != p && oe == e && e >= 0) { sum += oa; if (j < p) writes = false; }
    }
    if (writes && dense) {
      const float d = dm ? dm[e] * inv_s : 0.f;
      if (a.sigmoid) sum += d * sigmoid_f(l) / (1.f + expf(l));
      else sum += expf(l - mx) * inv * (d - dot);
    }
#pragma unroll
    for (int j = 0; j < V / W; ++j) {
      const int off = (j * LPR + p) * W;
      if (active && off < a.E) {
        float o[W];
#pragma unroll
        for (int w = 0; w < W; ++w) o[w] = 0.f;
        if (dense) {
          constexpr int C = W < 4 ? W : 4;
          float d[W];
#pragma unroll
          for (int w = 0; w < W; ++w) d[w] = 0.f;
          if (dm) {
#pragma unroll
            for (int w = 0; w < W; w += C) load_pack<float, C>(dm + off + w, d + w);
          }
#pragma unroll
          for (int w = 0; w < W; ++w) {
            const float x = v[j * W + w];
            if (a.sigmoid) o[w] = d[w] * inv_s * sigmoid_slope_fast(x);
            else o[w] = x * inv * (d[w] * inv_s - dot);
          }
        }
        store_pack<T, W>(out + off, o);
      }
    }
    __syncwarp();
    if (writes && active) out[e] = from_f32<T>(sum);
  }
}

template <typename T, int W, int LPR, int V, int MODE, bool MEAN>
bool launch_fwd_m(const RouteArgs& a, int G, float* sums, cudaStream_t st) {
  constexpr int regions = MEAN && V == 64 ? 2 : 1;
  constexpr int smem = regions * kRouteWarps * V * 32 * (int)sizeof(float);
  auto kern = route_fwd_fast_kernel<T, W, LPR, V, MODE, MEAN>;
  if (smem > 48 * 1024 && cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) {
    cudaGetLastError();
    return false;
  }
  kern<<<dim3(ceil_div(a.S, kRouteTile), G), kRouteThreads, smem, st>>>(a, sums);
  count_launch();
  return true;
}
template <typename T, int W, int LPR, int V>
bool launch_fwd(const RouteArgs& a, int G, float* sums, cudaStream_t st) {
#define GSHARD_ROUTE_MODE(MODE) \
  (sums ? launch_fwd_m<T, W, LPR, V, MODE, true>(a, G, sums, st) : launch_fwd_m<T, W, LPR, V, MODE, false>(a, G, sums, st))
  if (a.bias) return a.sigmoid ? GSHARD_ROUTE_MODE(kBySigmoidBias) : GSHARD_ROUTE_MODE(kBySoftmaxBias);
  if (a.groups > 1 && a.group_top == 2) return GSHARD_ROUTE_MODE(kBySums);
  return GSHARD_ROUTE_MODE(kByLogits);
#undef GSHARD_ROUTE_MODE
}
template <typename T, int W, int LPR, int V>
void launch_bwd(const RouteGradArgs& a, cudaStream_t st) {
  const long long blocks = (a.n + kRouteWarps * (32 / LPR) - 1) / (kRouteWarps * (32 / LPR));
  const int grid = (int)std::min<long long>(blocks, (long long)device_sms() * 64);
  route_bwd_fast_kernel<T, W, LPR, V><<<grid, kRouteThreads, 0, st>>>(a);
  count_launch();
}

// Values per lane (8, 16, 32 or 64) and lanes per token for E experts in `groups` groups; 0 = these kernels do
// not apply (more than 64 values per lane, or groups that lanes cannot share evenly).
struct RouteFit { int lpr, v; };
template <typename T>
RouteFit route_fit(int E, int groups, int k, long long n, int w) {
  RouteFit f{0, 0};
  if (groups & (groups - 1)) return f;
  for (int lpr : {8, 32}) {
    // few tokens: a token's latency counts, and a whole warp has it done sooner
    if (lpr == 8 && (groups > 8 || k > 8 || n < 148 * 16 || w == 1)) continue;
    const int per = lpr / groups * w;
    const int v = (E / groups + per - 1) / per * w;
    if (v > 64) continue;
    f.lpr = lpr; f.v = v <= 8 ? 8 : v <= 16 ? 16 : v <= 32 ? 32 : 64;
    break;
  }
  return f;
}

#define GSHARD_ROUTE_V(FN, LPR, W, ...)                                  \
  (f.v == 8 ? FN<T, W, LPR, 8>(__VA_ARGS__) : f.v == 16 ? FN<T, W, LPR, 16>(__VA_ARGS__) \
   : f.v == 32 ? FN<T, W, LPR, 32>(__VA_ARGS__) : FN<T, W, LPR, 64>(__VA_ARGS__))

}  // namespace

// sums: partial rows of the mean scores [G][tiles][E] (m itself where there is one tile), or nullptr.
// false = no kernel here fits the shape.
template <typename T>
bool launch_route_fwd_fast(const RouteArgs& a, int G, float* sums, cudaStream_t st) {
  constexpr int WF = 16 / (int)sizeof(T);
  const bool whole = a.E / a.groups % WF == 0;             // groups and rows in whole 16-byte words
  const RouteFit f = route_fit<T>(a.E, a.groups, a.k, a.n, whole ? WF : 1);
  if (!f.lpr) return false;
  if (!whole) return f.v <= 16 ? launch_fwd<T, 1, 32, 16>(a, G, sums, st) : launch_fwd<T, 1, 32, 64>(a, G, sums, st);
  if (f.lpr == 8) return GSHARD_ROUTE_V(launch_fwd, 8, WF, a, G, sums, st);
  return GSHARD_ROUTE_V(launch_fwd, 32, WF, a, G, sums, st);
}

template <typename T>
bool launch_route_bwd_fast(const RouteGradArgs& a, cudaStream_t st) {
  constexpr int WF = 16 / (int)sizeof(T);
  const bool whole = a.E % WF == 0;
  const RouteFit f = route_fit<T>(a.E, 1, a.k, a.n, whole ? WF : 1);
  if (!f.lpr) return false;
  if (!whole) f.v <= 16 ? launch_bwd<T, 1, 32, 16>(a, st) : launch_bwd<T, 1, 32, 64>(a, st);
  else if (f.lpr == 8) GSHARD_ROUTE_V(launch_bwd, 8, WF, a, st);
  else GSHARD_ROUTE_V(launch_bwd, 32, WF, a, st);
  return true;
}

}  // namespace gshard
