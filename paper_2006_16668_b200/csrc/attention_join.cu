// Cross attention: adds what the parts of a long axis have left, in order, one warp per (token, head).
#include "attention.cuh"
#include "pack.cuh"

namespace gshard {

namespace {

// o = sum of w_i o_i with w_i = 2^(lse_i) over their sum
template <typename T>
__global__ void __launch_bounds__(256) attention_join_kernel(const AttentionArgs a, const float* __restrict__ part_o,
                                                             const float* __restrict__ part_lse, int parts, long long rows) {
  const int lane = threadIdx.x & 31, c = lane * 4;
  for (long long r = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); r < rows; r += (long long)gridDim.x * 8) {
    float top = -INFINITY;
    for (int i = 0; i < parts; ++i) top = fmaxf(top, part_lse[i * rows + r]);
    const float ref = top == -INFINITY ? 0.f : top;
    float sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < parts; ++i) {
      const float lse = part_lse[i * rows + r];
      if (lse == -INFINITY) continue;          // no key in this part
      const float w = exp2f(lse - ref);
      sum += w;
      if (c < a.D) {
        const float4 x = *reinterpret_cast<const float4*>(part_o + (i * rows + r) * a.D + c);
        o[0] = fmaf(w, x.x, o[0]); o[1] = fmaf(w, x.y, o[1]); o[2] = fmaf(w, x.z, o[2]); o[3] = fmaf(w, x.w, o[3]);
      }
    }
    const long long token = r / a.H;
    const bool keys = source_length(a, (int)(token / a.Tq)) > 0;
    const float factor = keys ? 1.f / sum : 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] *= factor;
    if (c < a.D) store_pack<T, 4>(static_cast<T*>(a.o) + r * a.D + c, o);
    if (a.lse && lane == 0) {
      a.lse[((token / a.Tq) * a.H + r % a.H) * a.Tq + token % a.Tq] = !keys ? -INFINITY : (ref + log2f(sum)) * kLn2;
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(256) attention_join_gradient_kernel(const AttentionArgs a, const float* __restrict__ part, int parts,
                                                                      int part_keys, T* out, int tokens, int heads, long long stride,
                                                                      float factor, size_t pitch, long long rows) {
  const int c = (threadIdx.x & 31) * 4;
  for (long long r = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); r < rows; r += (long long)gridDim.x * 8) {
    const long long token = r / heads;
    const int b = (int)(token / tokens), t = (int)(token % tokens), len = source_length(a, b);
    const int there = part_keys ? min(parts, (len + part_keys - 1) / part_keys) : t < len ? parts : 0;
    if (c >= a.D) continue;
    float g[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < there; ++i) {
      const float4 x = *reinterpret_cast<const float4*>(part + i * pitch + r * a.D + c);
      g[0] += x.x; g[1] += x.y; g[2] += x.z; g[3] += x.w;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) g[j] *= factor;
    store_pack<T, 4>(out + token * stride + r % heads * a.D + c, g);
  }
}

}  // namespace

int launch_join_outputs(const AttentionArgs& a, bool bf16, const float* part_o, const float* part_lse, int parts, cudaStream_t st) {
  const long long rows = (long long)a.B * a.Tq * a.H;
  if (bf16) attention_join_kernel<__nv_bfloat16><<<grid_for_rows(rows), 256, 0, st>>>(a, part_o, part_lse, parts, rows);
  else attention_join_kernel<float><<<grid_for_rows(rows), 256, 0, st>>>(a, part_o, part_lse, parts, rows);
  count_launch();
  return cudaGetLastError() == cudaSuccess ? GSHARD_OK : GSHARD_ERR_CUDA;
}

int launch_join_gradient(const AttentionArgs& a, bool bf16, const float* part, int parts, int part_keys, void* out, int tokens, int heads,
                         long long stride, float factor, cudaStream_t st, size_t pitch) {
  const long long rows = (long long)a.B * tokens * heads;
  if (bf16)
    attention_join_gradient_kernel<<<grid_for_rows(rows), 256, 0, st>>>(a, part, parts, part_keys, static_cast<__nv_bfloat16*>(out), tokens, heads,
                                                                        stride, factor, pitch, rows);
  else
    attention_join_gradient_kernel<<<grid_for_rows(rows), 256, 0, st>>>(a, part, parts, part_keys, static_cast<float*>(out), tokens, heads, stride,
                                                                        factor, pitch, rows);
  count_launch();
  return cudaGetLastError() == cudaSuccess ? GSHARD_OK : GSHARD_ERR_CUDA;
}

}  // namespace gshard
