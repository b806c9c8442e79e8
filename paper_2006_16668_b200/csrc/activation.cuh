// Activations of the linear operator and their derivatives, in fp32.
#pragma once
#include "common.cuh"

namespace gshard {

// max(v, 0), where NaN stays NaN (fmaxf would answer 0)
__device__ __forceinline__ float relu(float v) {
  float y;
  asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(y) : "f"(v));
  return y;
}

// relu(v), v Phi(v) (erf form), its tanh approximation 0.5 v (1 + tanh(u)) = v / (1 + exp(-2u)) with
// u = sqrt(2/pi) (v + 0.044715 v^3), and v / (1 + exp(-v)).  exp may overflow to infinity: the quotient is then 0.
__device__ __forceinline__ float activation_value(float v, int act) {
  switch (act) {
    case GSHARD_ACT_RELU: return relu(v);
    case GSHARD_ACT_GELU: return 0.5f * v * (1.f + erff(v * 0.70710678118654752f));
    case GSHARD_ACT_GELU_TANH: return v / (1.f + expf(-1.5957691216057308f * v * fmaf(0.044715f * v, v, 1.f)));
    case GSHARD_ACT_SILU: return v / (1.f + expf(-v));
    default: return v;
  }
}

__device__ __forceinline__ float activation_slope(float v, int act) {
  switch (act) {
    case GSHARD_ACT_RELU: return v > 0.f ? 1.f : 0.f;
    case GSHARD_ACT_GELU:
      return fmaf(v * 0.39894228040143268f, expf(-0.5f * v * v), 0.5f * (1.f + erff(v * 0.70710678118654752f)));
    case GSHARD_ACT_GELU_TANH: {
      // with s = 1 / (1 + exp(-2u)): d(v s)/dv = s + v s (1 - s) d(2u)/dv.  s (1 - s) is 0 long before v^2 overflows,
      // and d(2u)/dv is held to a finite value so that the product stays 0.
      const float s = 1.f / (1.f + expf(-1.5957691216057308f * v * fmaf(0.044715f * v, v, 1.f)));
      return fmaf(v * s * (1.f - s), 1.5957691216057308f * fminf(fmaf(0.134145f * v, v, 1.f), 1e30f), s);
    }
    case GSHARD_ACT_SILU: {
      const float s = 1.f / (1.f + expf(-v));
      return s * fmaf(v, 1.f - s, 1.f);
    }
    default: return 1.f;
  }
}

// The same for results that are rounded to 16 bits: two approximate operations (2^x and 1/x, 1 to 2 units in the last
// place of fp32) instead of the library's exp, erf and division, which took longer than the matrix product they
// follow (65536 x 1024 x 8192 with gelu: 1409 us against 823 us without an activation).
__device__ __forceinline__ float approx_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float approx_rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Upper tail of the normal distribution, Phi(-|v|), by formula 7.1.26 of Abramowitz and Stegun (absolute error below
// 1e-7); e = exp(-v^2 / 2) comes out beside it.
__device__ __forceinline__ float normal_tail(float v, float& e) {
  const float a = fabsf(v);
  const float t = approx_rcp(fmaf(a, 0.3275911f * 0.70710678f, 1.f));
  e = approx_exp2(v * v * -0.72134752f);
  float p = fmaf(t, 0.5f * 1.061405429f, 0.5f * -1.453152027f);
  p = fmaf(t, p, 0.5f * 1.421413741f);
  p = fmaf(t, p, 0.5f * -0.284496736f);
  p = fmaf(t, p, 0.5f * 0.254829592f);
  return p * t * e;
}
__device__ __forceinline__ float activation_value_fast(float v, int act) {
  switch (act) {
    case GSHARD_ACT_RELU: return relu(v);
    case GSHARD_ACT_GELU: {
      float e;
      const float q = normal_tail(v, e);
      // v (1 - q) or v q; q is 0 from 14 on, and the product stays 0 for an infinite v
      return fmaf(-fabsf(fminf(v, 16.f)), q, fmaxf(v, 0.f));
    }
    case GSHARD_ACT_GELU_TANH: {
      const float d = 1.f + approx_exp2(-2.3022082f * v * fmaf(0.044715f * v, v, 1.f));
      return v * approx_rcp(d);
    }
    case GSHARD_ACT_SILU: return v * approx_rcp(1.f + approx_exp2(-1.4426950408889634f * v));
    default: return v;
  }
}
__device__ __forceinline__ float activation_slope_fast(float v, int act) {
  switch (act) {
    case GSHARD_ACT_RELU: return v > 0.f ? 1.f : 0.f;
    case GSHARD_ACT_GELU: {
      float e;
      const float q = normal_tail(v, e);
      return fmaf(v * 0.39894228040143268f, e, v > 0.f ? 1.f - q : q);
    }
    case GSHARD_ACT_GELU_TANH: {
      const float s = approx_rcp(1.f + approx_exp2(-2.3022082f * v * fmaf(0.044715f * v, v, 1.f)));
      return fmaf(v * s * (1.f - s), 1.5957691216057308f * fminf(fmaf(0.134145f * v, v, 1.f), 1e30f), s);
    }
    case GSHARD_ACT_SILU: {
      const float s = approx_rcp(1.f + approx_exp2(-1.4426950408889634f * v));
      return s * fmaf(v, 1.f - s, 1.f);
    }
    default: return 1.f;
  }
}

// N accumulator values (as register bits) in place; the branch on `act` is uniform and taken once.  FAST: the
// result is rounded to 16 bits.
template <int N, bool FAST>
__device__ __forceinline__ void activate(uint32_t* r, int act) {
#define GSHARD_ACT_LOOP(A)                                                                        \
  case A:                                                                                         \
    _Pragma("unroll") for (int i = 0; i < N; ++i)                                                 \
      r[i] = __float_as_uint(FAST ? activation_value_fast(__uint_as_float(r[i]), A)               \
                                  : activation_value(__uint_as_float(r[i]), A));                  \
    break;
  switch (act) {
    GSHARD_ACT_LOOP(GSHARD_ACT_RELU)
    GSHARD_ACT_LOOP(GSHARD_ACT_GELU)
    GSHARD_ACT_LOOP(GSHARD_ACT_GELU_TANH)
    GSHARD_ACT_LOOP(GSHARD_ACT_SILU)
    default: break;
  }
#undef GSHARD_ACT_LOOP
}

}  // namespace gshard
