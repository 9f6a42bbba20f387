// The activations of the layer operators and their derivatives, for device code compiled here (the generated kernels of the
// normalisation carry the same formulas in their own text).
#pragma once

#include <hip/hip_runtime.h>

#include "../../include/cgtp.h"

namespace cgtp {

// 1 / (1 + exp(-t)).  fp32: exp by the hardware's power of two, whose argument t log2(e) is corrected by its rounding error
// (without it the result is off by |t| roundings), and the hardware's reciprocal, 1 unit in the last place each.  Above 128 the
// result is 1; below -88, where it leaves the normal numbers, it is 0.  The selects keep a NaN, a clamp would not.
__device__ inline float act_sigmoid(float t) {
  const float s = t > 128.f ? 128.f : t;
  const float p = s * -1.44269502f;
  const float e = __builtin_fmaf(s, -1.44269502f, -p) + s * -1.92596299e-8f;
  const float x = __builtin_amdgcn_exp2f(p);
  const float q = __builtin_amdgcn_rcpf(1.f + __builtin_fmaf(x, 0.693147181f * e, x));
  return t < -88.f ? 0.f : q;
}
__device__ inline double act_sigmoid(double t) { return 1.0 / (1.0 + exp(-t)); }

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
    a = tanh(t);
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
