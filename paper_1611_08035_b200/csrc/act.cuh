// Activation functions and their derivatives, in fp32.
//
//   relu       max(z, 0)                                            0 or 1, 0 at z = 0
//   gelu       z Phi(z)                                             Phi(z) + z phi(z)
//   gelu_tanh  z s(2 u),  u = sqrt(2/pi) (z + 0.044715 z^3)         s + z s (1 - s) 2 u'        (tanh form: (1 + tanh u)/2 = s(2 u))
//   silu       z s(z),    s(x) = 1/(1 + exp(-x))                    s + z s (1 - s)
//
// exp and the reciprocal are the hardware's approximations (within 2^-22 relative); an argument of the exponential carries its own
// rounding, so that exp(-x) is within (1.5 x + 4) 2^-24 of itself.  Where the exponential is that far off, the function is next to 0 or the
// derivative next to its limit.  Infinite z gives the limits, NaN gives NaN.
//
// Phi: for x = |z|, Phi(-x) = exp(-x^2/2) t P(t) with t = 1/(1 + 0.3 x), P of degree 7 fitted to the scaled complementary error function
// (least largest relative error, 1.7e-7 for all x up to 14, where the exponential is 0 in single precision).  21 instructions with the
// exponential shared by the derivative.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "b2gemm.h"

namespace b2 {

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// bounds that keep NaN (fminf and fmaxf would drop it)
__device__ __forceinline__ float at_most(float x, float b) { return x > b ? b : x; }
__device__ __forceinline__ float at_least(float x, float b) { return x < b ? b : x; }

__device__ __forceinline__ float act_sigmoid(float x) { return rcp_approx(1.0f + exp2_approx(-1.44269504f * x)); }
// Phi(-x) for x >= 0, and exp(-x^2/2)
__device__ __forceinline__ float normal_tail(float x, float& e) {
  e = exp2_approx(-0.72134752f * (x * x));
  const float t = rcp_approx(fmaf(0.3f, x, 1.0f));
  float p = 0.03542371094226837f;
  p = fmaf(p, t, -0.15615835785865784f);
  p = fmaf(p, t, 0.2045566290616989f);
  p = fmaf(p, t, -0.05203389376401901f);
  p = fmaf(p, t, 0.12769171595573425f);
  p = fmaf(p, t, 0.10017596185207367f);
  p = fmaf(p, t, 0.12071213126182556f);
  p = fmaf(p, t, 0.11963200569152832f);
  return e * t * p;
}
constexpr float kGeluTanh = 0.7978845608f, kGeluCubic = 0.044715f;  // sqrt(2/pi)

template <int ACT>
__device__ __forceinline__ float act_value(float z) {
  if constexpr (ACT == B2_ACT_RELU) return z < 0.0f ? 0.0f : z;
  if constexpr (ACT == B2_ACT_GELU) {  // z > 0: z (1 - Phi(-z))
    float e;
    const float x = at_most(fabsf(z), 64.0f);
    return fmaf(-x, normal_tail(x, e), fmaxf(z, 0.0f));
  }
  if constexpr (ACT == B2_ACT_GELU_TANH) {
    const float x = at_most(at_least(z, -64.0f), 64.0f);
    return at_least(z, -64.0f) * act_sigmoid(2.0f * kGeluTanh * fmaf(kGeluCubic * x * x, x, x));
  }
  if constexpr (ACT == B2_ACT_SILU) {
    const float x = at_least(z, -200.0f);
    return x * act_sigmoid(x);
  }
  return z;
}
template <int ACT>
__device__ __forceinline__ float act_slope(float z) {
  if constexpr (ACT == B2_ACT_RELU) return z > 0.0f ? 1.0f : z <= 0.0f ? 0.0f : z;
  if constexpr (ACT == B2_ACT_GELU) {
    float e;
    const float x = at_most(at_least(z, -64.0f), 64.0f), h = normal_tail(fabsf(x), e);
    return fmaf(0.39894228f * x, e, x > 0.0f ? 1.0f - h : h);
  }
  if constexpr (ACT == B2_ACT_GELU_TANH) {
    const float x = at_most(at_least(z, -64.0f), 64.0f), x2 = x * x;
    const float s = act_sigmoid(2.0f * kGeluTanh * fmaf(kGeluCubic * x2, x, x));
    return fmaf(x * s * (1.0f - s), 2.0f * kGeluTanh * fmaf(3.0f * kGeluCubic, x2, 1.0f), s);
  }
  if constexpr (ACT == B2_ACT_SILU) {
    const float x = at_most(at_least(z, -200.0f), 200.0f), s = act_sigmoid(x);
    return fmaf(x * s, 1.0f - s, s);
  }
  return 1.0f;
}

// One test of the function for N numbers.
template <int ACT, int N>
__device__ __forceinline__ void act_values_of(float* v) {
#pragma unroll
  for (int j = 0; j < N; ++j) v[j] = act_value<ACT>(v[j]);
}
template <int N>
__device__ __forceinline__ void act_values(int act, float* v) {
  if (act == B2_ACT_RELU) act_values_of<B2_ACT_RELU, N>(v);
  else if (act == B2_ACT_GELU) act_values_of<B2_ACT_GELU, N>(v);
  else if (act == B2_ACT_GELU_TANH) act_values_of<B2_ACT_GELU_TANH, N>(v);
  else if (act == B2_ACT_SILU) act_values_of<B2_ACT_SILU, N>(v);
}
// v := v * act'(z)
template <int ACT, int N>
__device__ __forceinline__ void act_slopes_of(float* v, const float* z) {
#pragma unroll
  for (int j = 0; j < N; ++j) v[j] *= act_slope<ACT>(z[j]);
}
template <int N>
__device__ __forceinline__ void act_slopes(int act, float* v, const float* z) {
  if (act == B2_ACT_RELU) act_slopes_of<B2_ACT_RELU, N>(v, z);
  else if (act == B2_ACT_GELU) act_slopes_of<B2_ACT_GELU, N>(v, z);
  else if (act == B2_ACT_GELU_TANH) act_slopes_of<B2_ACT_GELU_TANH, N>(v, z);
  else if (act == B2_ACT_SILU) act_slopes_of<B2_ACT_SILU, N>(v, z);
}

inline bool act_known(int act) { return act >= B2_ACT_NONE && act <= B2_ACT_SILU; }

}  // namespace b2
