// The activations of the layer operators and their derivatives, for device code compiled here (the generated kernels of the
// normalisation carry the same formulas in their own text).
#pragma once

#include <hip/hip_runtime.h>

#include "../../include/cgtp.h"

namespace cgtp {

// 1 / (1 + exp(-t)).  fp32: the hardware's power of two and reciprocal.  The rounding of t log2(e) makes the result off by |t| half
// steps where t is negative, which is at most 0.3 half steps of 1, and t times it at most 0.6: a choice, which the header states.  With the argument
// corrected (five instructions more) the block of 160 710 x 64 x 2176 takes 497 us forward for 478 and 1992 backward for 1913, with 8 columns of x 281 for 274
// and 941 for 868.  No input leaves the range: 2^x gives infinity or zero, and the reciprocal zero or one.
__device__ inline float act_sigmoid(float t) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(t * -1.44269502f)); }
__device__ inline double act_sigmoid(double t) { return 1.0 / (1.0 + exp(-t)); }

// fp32: 1 - 2 / (1 + exp(2 |t|)), and near zero, where that loses bits, five terms of the series (the sixth is below 2^-27 of the result
// there).  Without branches: kernels whose registers overflow must not have lane-conditional code.
__device__ inline float act_tanh(float t) {
  const float s = t * t, x = __builtin_fabsf(t);
  const float p = t + t * s * (-0.333333333f + s * (0.133333333f + s * (-0.0539682540f + s * 0.0218694885f)));
  const float q = 1.f - 2.f * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * 2.88539008f));
  return x < 0.25f ? p : __builtin_copysignf(q, t);
}
__device__ inline double act_tanh(double t) { return tanh(t); }

// a = act(t) and d = act'(t)
template <int kAct, class T>
__device__ inline void act_both(T t, T& a, T& d) {
  if constexpr (kAct == CGTP_ACT_NONE) {
    a = t;
    d = T(1);
  } else if constexpr (kAct == CGTP_ACT_SILU) {
    const T q = act_sigmoid(t);
    a = t * q;
    d = q + a * (T(1) - q);
  } else if constexpr (kAct == CGTP_ACT_GELU) {
    const T p = T(0.5) * erfc(t * T(-0.70710678118654752440));
    a = t * p;
    d = p + t * (T(0.39894228040143267794) * exp(T(-0.5) * t * t));
  } else if constexpr (kAct == CGTP_ACT_SIGMOID) {
    a = act_sigmoid(t);
    d = a * (T(1) - a);
  } else {
    a = act_tanh(t);
    d = T(1) - a * a;
  }
}

template <int kAct, class T>
__device__ inline T act_only(T t) {
  T a, d;
  act_both<kAct>(t, a, d);
  return a;
}

}  // namespace cgtp
