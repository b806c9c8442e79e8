// W consecutive elements moved as one load or store (W * sizeof(T) bytes, naturally aligned), widened to fp32, and
// packed fp32 arithmetic.
#pragma once
#include "common.cuh"

namespace gshard {

template <int BYTES> struct RawWord;
template <> struct RawWord<16> { using type = uint4; };
template <> struct RawWord<8> { using type = uint2; };
template <> struct RawWord<4> { using type = unsigned; };
template <> struct RawWord<2> { using type = unsigned short; };

// One load's worth of elements as they lie in memory; get(j) widens element j.
template <typename T, int W> struct Pack {
  typename RawWord<W * (int)sizeof(T)>::type raw;
  __device__ __forceinline__ unsigned word(int i) const {
    if constexpr (W * sizeof(T) == 16) return i == 0 ? raw.x : i == 1 ? raw.y : i == 2 ? raw.z : raw.w;
    else if constexpr (W * sizeof(T) == 8) return i == 0 ? raw.x : raw.y;
    else return raw;
  }
  __device__ __forceinline__ float get(int j) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(word(j));
    else return __uint_as_float(j & 1 ? word(j / 2) & 0xffff0000u : word(j / 2) << 16);
  }
  __device__ __forceinline__ void load(const T* p) { raw = *reinterpret_cast<const decltype(raw)*>(p); }
  // for data read once: leaves L1 to what is read again
  __device__ __forceinline__ void load_once(const T* p) {
    if constexpr (W * sizeof(T) == 16)
      asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(raw.x), "=r"(raw.y), "=r"(raw.z), "=r"(raw.w) : "l"(p));
    else if constexpr (W * sizeof(T) == 8)
      asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(raw.x), "=r"(raw.y) : "l"(p));
    else if constexpr (W * sizeof(T) == 4)
      asm volatile("ld.global.L1::no_allocate.u32 %0, [%1];" : "=r"(raw) : "l"(p));
    else
      asm volatile("ld.global.L1::no_allocate.u16 %0, [%1];" : "=h"(raw) : "l"(p));
  }
};

template <typename T, int W>
__device__ __forceinline__ void load_pack(const T* p, float* f) {
  Pack<T, W> k;
  k.load(p);
#pragma unroll
  for (int j = 0; j < W; ++j) f[j] = k.get(j);
}
template <typename T, int W>
__device__ __forceinline__ void store_pack(T* p, const float* f) {
  unsigned w[4] = {0, 0, 0, 0};
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int j = 0; j < W; ++j) w[j] = __float_as_uint(f[j]);
  } else if constexpr (W == 1) {
    *p = __float2bfloat16_rn(f[0]);
    return;
  } else {
#pragma unroll
    for (int j = 0; j < W / 2; ++j) {
      const __nv_bfloat162 pr = __floats2bfloat162_rn(f[2 * j], f[2 * j + 1]);
      w[j] = *reinterpret_cast<const unsigned*>(&pr);
    }
  }
  if constexpr (W * sizeof(T) == 16) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  else if constexpr (W * sizeof(T) == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
  else *reinterpret_cast<unsigned*>(p) = w[0];
}

// Two fp32 values in a 64-bit register: two operations per instruction.
using f32x2 = unsigned long long;
__device__ __forceinline__ f32x2 pair(float lo, float hi) {
  f32x2 d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
  return d;
}
__device__ __forceinline__ float2 unpair(f32x2 v) {
  float2 f;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(v));
  return f;
}
__device__ __forceinline__ f32x2 both(float v) { return pair(v, v); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

}  // namespace gshard
