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
__device__ __forceinline__ float exp_minus(float v) {
  constexpr float REST = (float)(1.4426950408889634 - (double)LOG2E);
  const float m = v != v ? v : -__builtin_amdgcn_fmed3f(v, -200.0f, 200.0f);
  const float h = m * LOG2E;
  const float r = __builtin_fmaf(m, REST, __builtin_fmaf(m, LOG2E, -h));
  return __builtin_amdgcn_exp2f(h) * __builtin_fmaf(r, 0.6931471805599453f, 1.0f);
}
template <class E>
__device__ __forceinline__ float sigmoid(float v, float& e) {
  e = sizeof(E) == 2 ? __builtin_amdgcn_exp2f(-v * LOG2E) : exp_minus(v);
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

// softplus(lam) = max(lam, 0) + log(1 + e), e = e^-|lam|, to a few units of 2^-24: with w = 1 + e
// as rounded, log(1 + e) = log(w) e / (w - 1).  (The library's functions took some 200
// instructions of the first wave, which the others wait for.)
__device__ __forceinline__ float softplus(float lam, float& e) {
  e = exp_minus(fabsf(lam));
  const float w = 1.0f + e;
  const float l = __builtin_amdgcn_logf(w) * 0.6931471805599453f * (e * __builtin_amdgcn_rcpf(w - 1.0f));
  return fmaxf(lam, 0.0f) + (w == 1.0f ? e : l);
}
__device__ __forceinline__ float rate_of(float lam, float c) {
  float e;
  return c * softplus(lam, e);
}
// sigmoid(lam) / softplus(lam), which tends to 1 for lam -> -inf: below -16 it differs by
// e^lam / 2 < 2^-24.
__device__ __forceinline__ float rate_slope(float lam) {
  float e;
  const float p = softplus(lam, e);
  const float s = (lam > 0.0f ? 1.0f : e) * __builtin_amdgcn_rcpf(1.0f + e);
  return lam < -16.0f ? 1.0f : s * __builtin_amdgcn_rcpf(p);
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
