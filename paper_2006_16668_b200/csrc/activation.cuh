// Activations of the linear operator and their derivatives, in fp32.
#pragma once
#include "common.cuh"

namespace gshard {

// relu(v), v Phi(v) (erf form), its tanh approximation 0.5 v (1 + tanh(u)) = v / (1 + exp(-2u)) with
// u = sqrt(2/pi) (v + 0.044715 v^3), and v / (1 + exp(-v)).  exp may overflow to infinity: the quotient is then 0.
__device__ __forceinline__ float activation_value(float v, int act) {
  switch (act) {
    case GSHARD_ACT_RELU: return fmaxf(v, 0.f);
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
      // with s = 1 / (1 + exp(-2u)): d(v s)/dv = s + v s (1 - s) d(2u)/dv
      const float s = 1.f / (1.f + expf(-1.5957691216057308f * v * fmaf(0.044715f * v, v, 1.f)));
      return fmaf(v * s * (1.f - s), 1.5957691216057308f * fmaf(0.134145f * v, v, 1.f), s);
    }
    case GSHARD_ACT_SILU: {
      const float s = 1.f / (1.f + expf(-v));
      return s * fmaf(v, 1.f - s, 1.f);
    }
    default: return 1.f;
  }
}

// N accumulator values (as register bits) in place; the branch on `act` is uniform and taken once.
template <int N>
__device__ __forceinline__ void activate(uint32_t* r, int act) {
#define GSHARD_ACT_LOOP(A)                                                                        \
  case A:                                                                                         \
    _Pragma("unroll") for (int i = 0; i < N; ++i)                                                 \
      r[i] = __float_as_uint(activation_value(__uint_as_float(r[i]), A));                         \
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
