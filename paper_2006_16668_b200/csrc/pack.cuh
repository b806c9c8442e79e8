// W consecutive elements moved as one load or store (W * sizeof(T) bytes, naturally aligned), widened to fp32.
#pragma once
#include "common.cuh"

namespace gshard {

template <typename T, int W> struct alignas(sizeof(T) * W) Pack { T v[W]; };

template <typename T, int W>
__device__ __forceinline__ void load_pack(const T* p, float* f) {
  const Pack<T, W> k = *reinterpret_cast<const Pack<T, W>*>(p);
#pragma unroll
  for (int j = 0; j < W; ++j) f[j] = to_f32<T>(k.v[j]);
}
template <typename T, int W>
__device__ __forceinline__ void store_pack(T* p, const float* f) {
  Pack<T, W> k;
#pragma unroll
  for (int j = 0; j < W; ++j) k.v[j] = from_f32<T>(f[j]);
  *reinterpret_cast<Pack<T, W>*>(p) = k;
}

}  // namespace gshard
