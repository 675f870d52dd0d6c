// gated_math.h -- the gates of the recurrence (device code).
//
//   m = k sigmoid(r),  k = c softplus(lam),  a = e^-m,  z = 1 - a^2,  u = sqrt(z) sigmoid(i) x
//
// z is formed from t = 2 m: below a bound as the series of 1 - e^-t, which keeps its
// digits as a nears 1 (a channel with a long memory), above it as 1 - a a, whose
// subtraction loses none that matter there: at the bound 2^-24 / z is 2^-21 for bf16
// inputs and 2^-22 for fp32 ones, and the square root halves it.
#pragma once

#include "sw_internal.h"

// Which products are fused is written out: the same in every instance, whatever its loads.
#pragma clang fp contract(off)

namespace sw {
namespace gated {

constexpr float LOG2E = 1.4426950408889634f;

// 1 / (1 + e^-v), and e = e^-v (infinite below -88).  fp32 inputs: the rounding of v
// log2 e, which alone would cost 2^-24 |v| of e, is made up for; v is held where e is
// 0 or infinite already, since an infinite one would make the correction NaN.
template <class E>
__device__ __forceinline__ float sigmoid(float v, float& e) {
  if constexpr (sizeof(E) == 2) {
    e = __builtin_amdgcn_exp2f(-v * LOG2E);
  } else {
    constexpr float REST = (float)(1.4426950408889634 - (double)LOG2E);
    const float m = v != v ? v : -__builtin_amdgcn_fmed3f(v, -200.0f, 200.0f);
    const float h = m * LOG2E;
    const float r = __builtin_fmaf(m, REST, __builtin_fmaf(m, LOG2E, -h));
    e = __builtin_amdgcn_exp2f(h) * __builtin_fmaf(r, 0.6931471805599453f, 1.0f);
  }
  return __builtin_amdgcn_rcpf(1.0f + e);
}
// 1 minus it, e s, which keeps its digits where s nears 1.  (An infinite e leaves 1; so does
// a NaN, which s hands on.)
__device__ __forceinline__ float sigmoid_rest(float e, float s) { return fminf(e * s, 1.0f); }

template <class E>
__device__ __forceinline__ float one_minus_square(float m, float a) {
  const float rest = __builtin_fmaf(-a, a, 1.0f);
  if constexpr (sizeof(E) == 2) {  // to t^4 / 120 of the value: 2^-19 at the bound
    float p = __builtin_fmaf(m, -2.0f / 3.0f, 4.0f / 3.0f);
    p = __builtin_fmaf(-m, p, 2.0f);
    p = m * __builtin_fmaf(-m, p, 2.0f);
    return m < 0.0625f ? p : rest;
  } else {  // to t^8 / 9!: 2^-26
    const float t = m + m;
    float p = __builtin_fmaf(t, -1.0f / 40320.0f, 1.0f / 5040.0f);
    p = __builtin_fmaf(-t, p, 1.0f / 720.0f);
    p = __builtin_fmaf(-t, p, 1.0f / 120.0f);
    p = __builtin_fmaf(-t, p, 1.0f / 24.0f);
    p = __builtin_fmaf(-t, p, 1.0f / 6.0f);
    p = __builtin_fmaf(-t, p, 0.5f);
    p = t * __builtin_fmaf(-t, p, 1.0f);
    return m < 0.25f ? p : rest;
  }
}

// c softplus(lam).
__device__ __forceinline__ float rate_of(float lam, float c) {
  return c * (fmaxf(lam, 0.0f) + log1pf(expf(-fabsf(lam))));
}
// sigmoid(lam) / softplus(lam), which tends to 1 for lam -> -inf: below -16 it differs by
// e^lam / 2 < 2^-24.
__device__ __forceinline__ float rate_slope(float lam) {
  if (lam < -16.0f) return 1.0f;
  const float e = expf(-fabsf(lam));
  const float s = lam > 0.0f ? 1.0f / (1.0f + e) : e / (1.0f + e);
  return s / (fmaxf(lam, 0.0f) + log1pf(e));
}

// A step's pair (a, u).
template <class E>
__device__ __forceinline__ void pair_of(float x, float r, float i, float k, float& a, float& u) {
  float e;
  const float m = k * sigmoid<E>(r, e);
  a = __builtin_amdgcn_exp2f(-m * LOG2E);
  u = __builtin_amdgcn_sqrtf(one_minus_square<E>(m, a)) * sigmoid<E>(i, e) * x;
}

// What a step's gradients need.
struct Step {
  float a, bs, q, ma;    // bs = b s, q = (m / b) a^2 s x, ma = m a, with s = sigmoid(i)
  float rest_r, rest_i;  // 1 - sigmoid(r), 1 - s
};
// An infinite m is held where a is zero, so that m a is; a z below 2^-122, where 1 / b would
// be infinite: both products end there as their limits do, at zero.  (A NaN that a minimum or
// maximum drops is in a or z still.)
template <class E>
__device__ __forceinline__ Step step_of(float x, float r, float i, float k) {
  Step t;
  float e;
  const float sr = sigmoid<E>(r, e);
  t.rest_r = sigmoid_rest(e, sr);
  const float m = k * sr;
  t.a = __builtin_amdgcn_exp2f(-m * LOG2E);
  const float z = one_minus_square<E>(m, t.a);
  const float inv = __builtin_amdgcn_rsqf(fmaxf(z, 1e-37f));
  const float si = sigmoid<E>(i, e);
  t.rest_i = sigmoid_rest(e, si);
  t.bs = z * inv * si;
  t.ma = fminf(m, 1e3f) * t.a;
  t.q = t.ma * t.a * inv * (si * x);
  return t;
}

}  // namespace gated
}  // namespace sw
