// Routing of tokens to experts beyond Algorithm 1's top-2 softmax gate: scores, a balancing bias that
// moves the choice but not the weights, choice inside the best groups of experts, k experts per token.
//
//   score      s_e = softmax(l)_e or sigmoid(l_e); a logit of -inf or NaN bars the expert for the token
//   choice     by c_e = s_e + b_e, larger first, equal values to the lowest index; with groups only the
//              experts of the best `groups_kept` groups compete (group value: its best c, or the sum of its
//              two best).  Without a bias the logits are compared instead: s grows with l.
//   weight     w_i = scale s_i, or scale s_i / sum of the chosen s
//   statistics m_{g,e} = (1/S) sum of s_e over the group's tokens (what Algorithm 1's l_aux takes), and
//              how many tokens of the group chose the expert (what moves a balancing bias)
//
// One warp per token.  Near ties between fp32 values of c would make the choice depend on rounding, so
// c is compared in 64 bits.
#include <algorithm>

#include "plan.cuh"
#include "route.cuh"

namespace gshard {

namespace {

template <typename T>
__global__ void __launch_bounds__(256) route_fwd_kernel(const __grid_constant__ RouteArgs a) {
  const int lane = threadIdx.x & 31;
  const long long nwarps = ((long long)gridDim.x * blockDim.x) >> 5;
  for (long long t = ((long long)blockIdx.x * blockDim.x + threadIdx.x) >> 5; t < a.n; t += nwarps) {
    const T* row = static_cast<const T*>(a.logits) + t * a.E;
    const int e = choose_exact<T>(row, a, lane, nullptr);
    float mx = 0.f, inv = 0.f;
    if (!a.sigmoid && (a.rowstat || !a.renorm)) {
      mx = -INFINITY;
      for (int i = lane; i < a.E; i += 32) mx = fmaxf(mx, usable(row[i]));
      mx = warp_max(mx);
      if (mx == -INFINITY) mx = 0.f;
      float s = 0.f;
      for (int i = lane; i < a.E; i += 32) s += expf(usable(row[i]) - mx);
      s = warp_sum(s);
      inv = s > 0.f ? 1.f / s : 0.f;
      if (a.rowstat && lane == 0) { a.rowstat[2 * t] = mx; a.rowstat[2 * t + 1] = inv; }
    }
    const float l = e >= 0 ? usable(row[e]) : -INFINITY;
    float w;
    if (a.renorm) {
      float total;
      w = chosen_ratio(l, a.sigmoid, total);
      w = total > 0.f ? a.scale * (w / total) : 0.f;
    } else {
      w = e < 0 ? 0.f : a.scale * (a.sigmoid ? sigmoid_f(l) : expf(l - mx) * inv);
    }
    if (lane < a.k) {
      a.expert_idx[t * a.k + lane] = e;
      a.weight[t * a.k + lane] = w;
      if (a.load && e >= 0) atomicAdd(a.load + t / a.S * a.E + e, 1);
    }
  }
}

// partial[g][tile][e] = sum of s_e over the tile's tokens.  Thread = expert; grid (E / 128, tiles, G).
template <typename T>
__global__ void __launch_bounds__(128) route_colsum_kernel(const T* __restrict__ logits, const float* __restrict__ rowstat,
                                                           float* __restrict__ partial, int S, int E, int sigmoid) {
  const int e = blockIdx.x * 128 + threadIdx.x;
  if (e >= E) return;
  const long long tiles = gridDim.y;
  const int s0 = blockIdx.y * kRouteTile, s1 = min(S, s0 + kRouteTile);
  float sum = 0.f;
  for (int s = s0; s < s1; ++s) {
    const long long t = (long long)blockIdx.z * S + s;
    const float l = usable(logits[t * E + e]);
    sum += sigmoid ? sigmoid_f(l) : expf(l - rowstat[2 * t]) * rowstat[2 * t + 1];
  }
  partial[((long long)blockIdx.z * tiles + blockIdx.y) * E + e] = sum;
}

// m[g][e] = (1/S) sum over the tiles: 8 strands of tiles in order, then the strands.
__global__ void __launch_bounds__(256) route_mean_kernel(const float* __restrict__ partial, float* __restrict__ m, int tiles,
                                                         int S, int E) {
  __shared__ float part[8][33];
  const int e = blockIdx.x * 32 + threadIdx.x;
  float s = 0.f;
  if (e < E)
    for (int i = threadIdx.y; i < tiles; i += 8) s += partial[((long long)blockIdx.y * tiles + i) * E + e];
  part[threadIdx.y][threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.y == 0 && e < E) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += part[i][threadIdx.x];
    m[(long long)blockIdx.y * E + e] = s / (float)S;
  }
}

// Gradient of sum(dweight w) + sum(dm m) with the choice held constant.  With D = sum_j dw_j w_j / scale:
//   renormalised   d/dlog s_i = scale w_i (dw_i - D), so dl_i gets that (softmax), times 1 - s_i (sigmoid)
//   otherwise      d/ds_i = scale dw_i;  dm adds dm_e / S to every d/ds_e
//   softmax        dl_e += s_e (ds_e - sum_e' s_e' ds_e');  sigmoid: dl_e += ds_e s_e (1 - s_e)
// An index named twice by the caller receives the sum of its entries.
template <typename T>
__global__ void __launch_bounds__(256) route_bwd_kernel(const RouteGradArgs a) {
  const int lane = threadIdx.x & 31;
  const long long nwarps = ((long long)gridDim.x * blockDim.x) >> 5;
  const bool soft_stats = !a.sigmoid && (a.dm || !a.renorm);
  const float inv_s = 1.f / (float)a.S;
  for (long long t = ((long long)blockIdx.x * blockDim.x + threadIdx.x) >> 5; t < a.n; t += nwarps) {
    const T* row = static_cast<const T*>(a.logits) + t * a.E;
    T* out = static_cast<T*>(a.dlogits) + t * a.E;
    const float* dm = a.dm ? a.dm + t / a.S * a.E : nullptr;
    float mx = -INFINITY, inv = 0.f, dot = 0.f;
    if (soft_stats) {
      for (int i = lane; i < a.E; i += 32) mx = fmaxf(mx, usable(row[i]));
      mx = warp_max(mx);
      if (mx == -INFINITY) mx = 0.f;
      float s = 0.f;
      for (int i = lane; i < a.E; i += 32) s += expf(usable(row[i]) - mx);
      s = warp_sum(s);
      inv = s > 0.f ? 1.f / s : 0.f;
    }
    int e = -1;
    float l = -INFINITY, dw = 0.f;
    if (lane < a.k) {
      e = a.expert_idx[t * a.k + lane];
      if (e < 0 || e >= a.E) e = -1;
      if (e >= 0) { l = usable(row[e]); dw = a.dweight[t * a.k + lane]; }
      if (l == -INFINITY) e = -1;
    }
    float add = 0.f;                        // this entry's share of dl at its expert
    if (a.renorm) {
      float total;
      const float r = chosen_ratio(l, a.sigmoid, total);
      const float w = total > 0.f ? r / total : 0.f;
      const float D = warp_sum(e >= 0 ? w * dw : 0.f);
      add = e >= 0 ? a.scale * w * (dw - D) : 0.f;
      if (a.sigmoid && e >= 0) add /= 1.f + expf(l);
    } else if (e >= 0) {
      const float s = a.sigmoid ? sigmoid_f(l) : expf(l - mx) * inv;
      add = a.scale * dw * s;
      if (a.sigmoid) add /= 1.f + expf(l);
    }
    if (!a.sigmoid) {
      if (dm)
        for (int i = lane; i < a.E; i += 32) dot = fmaf(expf(usable(row[i]) - mx) * inv, dm[i] * inv_s, dot);
      dot = warp_sum(dot + (a.renorm ? 0.f : add));
    }
    auto dense = [&](int i) -> float {
      if (!soft_stats && !dm) return 0.f;
      const float li = usable(row[i]);
      if (li == -INFINITY) return 0.f;
      const float d = dm ? dm[i] * inv_s : 0.f;
      if (a.sigmoid) return d * sigmoid_f(li) / (1.f + expf(li));
      return expf(li - mx) * inv * (d - dot);
    };
    // entries that name the same expert add up; the first of them writes
    float sum = add;
    bool first = e >= 0;
    for (int j = 0; j < a.k; ++j) {
      const int oe = __shfl_sync(kAll, e, j);
      const float oa = __shfl_sync(kAll, add, j);
      if (j != lane && oe == e && e >= 0) { sum += oa; if (j < lane) first = false; }
    }
    const float mine = first ? dense(e) + sum : 0.f;
    for (int i = lane; i < a.E; i += 32) out[i] = from_f32<T>(dense(i));
    __syncwarp();
    if (first) out[e] = from_f32<T>(mine);
  }
}

struct RoutePlan { int tiles; size_t rowstat, partial, total; };
RoutePlan route_plan(const gshard_route_config& c) {
  Carver w;
  RoutePlan p;
  p.tiles = ceil_div(c.S, kRouteTile);
  p.rowstat = w.take((size_t)c.G * c.S * 2 * sizeof(float));
  p.partial = w.take((size_t)c.G * p.tiles * c.E * sizeof(float));
  p.total = w.off;
  return p;
}

int route_validate(const gshard_route_config* c) {
  if (!c || c->G < 0 || c->S < 0 || c->E <= 0 || c->k <= 0 || c->k > c->E) return GSHARD_ERR_INVALID_ARG;
  if (c->dtype != GSHARD_F32 && c->dtype != GSHARD_BF16) return GSHARD_ERR_INVALID_ARG;
  if (c->score != GSHARD_SCORE_SOFTMAX && c->score != GSHARD_SCORE_SIGMOID) return GSHARD_ERR_INVALID_ARG;
  if (c->groups < 1 || c->E % c->groups || c->groups_kept < 1 || c->groups_kept > c->groups) return GSHARD_ERR_INVALID_ARG;
  if (c->group_top != 1 && c->group_top != 2) return GSHARD_ERR_INVALID_ARG;
  if (c->k > c->groups_kept * (c->E / c->groups)) return GSHARD_ERR_INVALID_ARG;
  if (!std::isfinite(c->scale)) return GSHARD_ERR_INVALID_ARG;
  if (c->E > 16384 || c->k > kRouteMaxK || c->groups > kRouteMaxGroups) return GSHARD_ERR_UNSUPPORTED_SHAPE;
  if ((long long)c->G * c->S > (1ll << 30) || c->G > 65535 || ceil_div(c->S, kRouteTile) > 65535) return GSHARD_ERR_UNSUPPORTED_SHAPE;
  return GSHARD_OK;
}

}  // namespace

}  // namespace gshard

using namespace gshard;

extern "C" {

size_t gshard_moe_route_workspace_bytes(const gshard_route_config* config) {
  if (route_validate(config) != GSHARD_OK) return 0;
  const size_t n = route_plan(*config).total;
  return n ? n : kAlign;
}

int gshard_moe_route(const gshard_route_config* config, const void* logits, const float* bias, int32_t* expert_idx,
                     float* weight, float* m, int32_t* load, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  launch_counter().n = 0;
  GS_CHECK(route_validate(config));
  const gshard_route_config& c = *config;
  GS_CHECK_OPTIONAL_PTR(bias); GS_CHECK_OPTIONAL_PTR(m); GS_CHECK_OPTIONAL_PTR(load);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const long long n = (long long)c.G * c.S;
  if (n == 0) {                                   // no tokens: empty sums
    if (!c.G || (!m && !load)) return GSHARD_OK;
    GS_CHECK(check_device());
    if (m && cudaMemsetAsync(m, 0, (size_t)c.G * c.E * 4, st) != cudaSuccess) { cudaGetLastError(); return GSHARD_ERR_CUDA; }
    if (load && cudaMemsetAsync(load, 0, (size_t)c.G * c.E * 4, st) != cudaSuccess) { cudaGetLastError(); return GSHARD_ERR_CUDA; }
    return GSHARD_OK;
  }
  GS_CHECK_PTR(logits); GS_CHECK_PTR(expert_idx); GS_CHECK_PTR(weight);
  const RoutePlan pl = route_plan(c);
  if (m) GS_CHECK_WORKSPACE(workspace, workspace_bytes, pl.total);
  GS_CHECK(check_device());
  NvtxRange range("gshard.route");
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  RouteArgs a{};
  a.logits = logits; a.bias = bias; a.expert_idx = expert_idx; a.weight = weight; a.load = load;
  a.rowstat = m ? reinterpret_cast<float*>(ws + pl.rowstat) : nullptr;
  a.n = n; a.S = c.S; a.E = c.E; a.k = c.k; a.groups = c.groups; a.kept = c.groups_kept; a.group_top = c.group_top;
  a.sigmoid = c.score == GSHARD_SCORE_SIGMOID; a.renorm = c.renormalise != 0; a.scale = c.scale;
  if (load && cudaMemsetAsync(load, 0, (size_t)c.G * c.E * 4, st) != cudaSuccess) { cudaGetLastError(); return GSHARD_ERR_CUDA; }
  // kept == groups leaves nothing out
  if (a.kept == a.groups) a.groups = a.kept = 1;
  float* partial = m ? reinterpret_cast<float*>(ws + pl.partial) : nullptr;
  float* sums = pl.tiles == 1 ? m : partial;
  const bool bf16 = c.dtype == GSHARD_BF16;
  if (bf16 ? launch_route_fwd_fast<__nv_bfloat16>(a, c.G, sums, st) : launch_route_fwd_fast<float>(a, c.G, sums, st)) {
    if (m && pl.tiles > 1) {
      route_mean_kernel<<<dim3(ceil_div(c.E, 32), c.G), dim3(32, 8), 0, st>>>(partial, m, pl.tiles, c.S, c.E);
      count_launch();
    }
    return cudaGetLastError() == cudaSuccess ? GSHARD_OK : GSHARD_ERR_CUDA;
  }
  const int grid = grid_for_rows(n);
  if (bf16) route_fwd_kernel<__nv_bfloat16><<<grid, 256, 0, st>>>(a);
  else route_fwd_kernel<float><<<grid, 256, 0, st>>>(a);
  count_launch();
  if (m) {
    const dim3 cg(ceil_div(c.E, 128), pl.tiles, c.G);
    if (bf16)
      route_colsum_kernel<__nv_bfloat16><<<cg, 128, 0, st>>>(static_cast<const __nv_bfloat16*>(logits), a.rowstat, partial, c.S, c.E, a.sigmoid);
    else
      route_colsum_kernel<float><<<cg, 128, 0, st>>>(static_cast<const float*>(logits), a.rowstat, partial, c.S, c.E, a.sigmoid);
    route_mean_kernel<<<dim3(ceil_div(c.E, 32), c.G), dim3(32, 8), 0, st>>>(partial, m, pl.tiles, c.S, c.E);
    count_launch(2);
  }
  return cudaGetLastError() == cudaSuccess ? GSHARD_OK : GSHARD_ERR_CUDA;
}

int gshard_moe_route_backward(const gshard_route_config* config, const void* logits, const int32_t* expert_idx,
                              const float* dweight, const float* dm, void* dlogits, void* cuda_stream) {
  launch_counter().n = 0;
  GS_CHECK(route_validate(config));
  const gshard_route_config& c = *config;
  const long long n = (long long)c.G * c.S;
  if (n == 0) return GSHARD_OK;
  GS_CHECK_PTR(logits); GS_CHECK_PTR(expert_idx); GS_CHECK_PTR(dweight); GS_CHECK_PTR(dlogits);
  GS_CHECK_OPTIONAL_PTR(dm);
  if (dlogits == logits) return GSHARD_ERR_INVALID_ARG;     // chosen logits are read again after a row's first writes
  GS_CHECK(check_device());
  NvtxRange range("gshard.route.backward");
  RouteGradArgs a{};
  a.logits = logits; a.expert_idx = expert_idx; a.dweight = dweight; a.dm = dm; a.dlogits = dlogits;
  a.n = n; a.S = c.S; a.E = c.E; a.k = c.k; a.sigmoid = c.score == GSHARD_SCORE_SIGMOID; a.renorm = c.renormalise != 0;
  a.scale = c.scale;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const bool bf16 = c.dtype == GSHARD_BF16;
  if (!(bf16 ? launch_route_bwd_fast<__nv_bfloat16>(a, st) : launch_route_bwd_fast<float>(a, st))) {
    const int grid = grid_for_rows(n);
    if (bf16) route_bwd_kernel<__nv_bfloat16><<<grid, 256, 0, st>>>(a);
    else route_bwd_kernel<float><<<grid, 256, 0, st>>>(a);
    count_launch();
  }
  return cudaGetLastError() == cudaSuccess ? GSHARD_OK : GSHARD_ERR_CUDA;
}

}  // extern "C"
