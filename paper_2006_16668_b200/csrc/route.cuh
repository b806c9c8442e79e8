// Shared by the routing kernels: arguments, warp helpers, and the choice of one token in 64 bits.
#pragma once
#include <cfloat>
#include <climits>
#include <cmath>

#include "checks.cuh"
#include "pack.cuh"

namespace gshard {

constexpr int kRouteMaxK = 32;
constexpr int kRouteMaxGroups = 32;
constexpr int kRouteTile = 64;              // tokens per partial row of the mean scores
constexpr unsigned kAll = 0xffffffffu;

struct RouteArgs {
  const void* logits;
  const float* bias;
  int32_t* expert_idx;
  float* weight;
  float* rowstat;        // [N][2] softmax maximum and 1 / sum (for the mean scores), or nullptr
  int32_t* load;         // [G][E] or nullptr
  long long n;
  int S, E, k, groups, kept, group_top, sigmoid, renorm;
  float scale;
};

// NaN bars like -inf; +inf counts as the largest float, so that differences of logits stay finite.
template <typename T> __device__ __forceinline__ float usable(T v) {
  const float f = to_f32<T>(v);
  return f == f ? fminf(f, FLT_MAX) : -INFINITY;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor_sync(kAll, v, off));
  return v;
}
template <typename F> __device__ __forceinline__ F warp_sum(F v) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(kAll, v, off);
  return v;
}
// larger value first, equal values to the lower index
__device__ __forceinline__ void warp_best(double& v, int& e) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    const double ov = __shfl_xor_sync(kAll, v, off);
    const int oe = __shfl_xor_sync(kAll, e, off);
    if (ov > v || (ov == v && oe < e)) { v = ov; e = oe; }
  }
}

// The choice of one token in 64 bits: lane j < k receives the j-th expert (-1: none left).  cache: E doubles
// of the warp's shared memory for the values, or nullptr (they are then computed wherever they are needed).
template <typename T>
__device__ __noinline__ int choose_exact(const T* __restrict__ row, const RouteArgs& a, int lane, double* cache) {
  const bool scores = a.bias != nullptr || (a.groups > 1 && a.group_top == 2);
  double top = 0.0, inv = 1.0;
  if (scores && !a.sigmoid) {
    float mx = -INFINITY;
    for (int e = lane; e < a.E; e += 32) mx = fmaxf(mx, usable(row[e]));
    mx = warp_max(mx);
    top = mx == -INFINITY ? 0.0 : (double)mx;
    double s = 0.0;
    for (int e = lane; e < a.E; e += 32) s += exp((double)usable(row[e]) - top);
    s = warp_sum(s);
    inv = s > 0.0 ? s : 1.0;
  }
  auto value = [&](int e, bool by_score) -> double {
    const float l = usable(row[e]);
    if (l == -INFINITY) return -INFINITY;
    if (!by_score) return (double)l;
    const double s = a.sigmoid ? 1.0 / (1.0 + exp(-(double)l)) : exp((double)l - top) / inv;
    const double c = a.bias ? s + (double)a.bias[e] : s;
    return c == c ? c : -INFINITY;
  };
  // scores, or scores plus bias: what groups are valued by, and with a bias what the choice goes by
  if (cache && scores) {
    __syncwarp();
    for (int e = lane; e < a.E; e += 32) cache[e] = value(e, true);
    __syncwarp();
  }
  auto look = [&](int e, bool by_score) -> double { return cache && by_score ? cache[e] : value(e, by_score); };
  unsigned keep = kAll;
  const int size = a.E / a.groups;
  if (a.kept < a.groups) {
    double mine = -INFINITY;                    // lane g: the value of group g
    for (int g = 0; g < a.groups; ++g) {
      double b1 = -INFINITY, b2 = -INFINITY;
      for (int i = lane; i < size; i += 32) {
        const double v = look(g * size + i, scores);
        if (v > b1) { b2 = b1; b1 = v; } else if (v > b2) b2 = v;
      }
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) {
        const double o1 = __shfl_xor_sync(kAll, b1, off), o2 = __shfl_xor_sync(kAll, b2, off);
        if (o1 > b1) { b2 = fmax(b1, o2); b1 = o1; } else b2 = fmax(b2, o1);
      }
      const double v = (a.group_top == 2 && b2 != -INFINITY) ? b1 + b2 : b1;
      if (lane == g) mine = v;
    }
    keep = 0;
    bool taken = lane >= a.groups;
    for (int j = 0; j < a.kept; ++j) {
      double v = taken ? -INFINITY : mine;
      int e = taken ? 64 + lane : lane;
      warp_best(v, e);
      if (e < 32) keep |= 1u << e;
      if (e == lane) taken = true;
    }
  }
  int picked = -1;
  double last = INFINITY;
  int last_e = -1;
  for (int j = 0; j < a.k; ++j) {
    double best = -INFINITY;
    int at = INT_MAX;
    for (int e = lane; e < a.E; e += 32) {
      if (!((keep >> (e / size)) & 1u)) continue;
      const double v = look(e, a.bias != nullptr);
      if (v == -INFINITY || v > last || (v == last && e <= last_e)) continue;
      if (v > best || at == INT_MAX) { best = v; at = e; }
    }
    warp_best(best, at);
    if (at == INT_MAX) break;
    if (lane == j) picked = at;
    last = best; last_e = at;
  }
  if (cache) __syncwarp();
  return picked;
}

// Lane j holds chosen expert idx (or -1) with logit l (or -inf): its score over the largest chosen score, and
// the sum of those ratios over the warp.  Stays exact where the scores themselves underflow.
__device__ __forceinline__ float chosen_ratio(float l, int sigmoid, float& total) {
  float top = warp_max(l);
  if (top == -INFINITY) top = 0.f;
  float r;
  if (!sigmoid) r = expf(l - top);
  else if (top < 0.f) r = expf(l - top) * (1.f + expf(top)) / (1.f + expf(fminf(l, 0.f)));
  else r = (1.f + expf(-top)) / (1.f + expf(-l));
  if (l == -INFINITY) r = 0.f;
  total = warp_sum(r);
  return r;
}
__device__ __forceinline__ float sigmoid_f(float l) { return 1.f / (1.f + expf(-l)); }

struct RouteGradArgs {
  const void* logits;
  const int32_t* expert_idx;
  const float* dweight;
  const float* dm;       // [G][E] or nullptr
  void* dlogits;
  long long n;
  int S, E, k, sigmoid, renorm;
  float scale;
};

// route_fast.cuh
template <typename T> bool launch_route_fwd_fast(const RouteArgs& a, int G, float* sums, cudaStream_t st);
template <typename T> bool launch_route_bwd_fast(const RouteGradArgs& a, cudaStream_t st);

}  // namespace gshard
