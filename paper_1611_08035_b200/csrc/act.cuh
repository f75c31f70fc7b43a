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
// (least largest relative error, 1.7e-7 for all x up to 14, where the exponential is 0 in single precision).
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
__device__ __forceinline__ float at_most(float x, float b) {
  float y;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(x), "f"(b));
  return y;
}
__device__ __forceinline__ float at_least(float x, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(x), "f"(b));
  return y;
}

__device__ __forceinline__ float larger_nan(float a, float b) { return at_least(a, b); }

// Two numbers at a time: the packed fp32 instructions do both for one.
struct Two {
  float a, b;
};
__device__ __forceinline__ uint64_t bits_of(Two x) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(x.a), "f"(x.b));
  return d;
}
__device__ __forceinline__ Two two_of(uint64_t d) {
  Two x;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(x.a), "=f"(x.b) : "l"(d));
  return x;
}
__device__ __forceinline__ Two both(float x) { return {x, x}; }
__device__ __forceinline__ Two fma2(Two x, Two y, Two z) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(bits_of(x)), "l"(bits_of(y)), "l"(bits_of(z)));
  return two_of(d);
}
__device__ __forceinline__ Two mul2(Two x, Two y) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(bits_of(x)), "l"(bits_of(y)));
  return two_of(d);
}
__device__ __forceinline__ Two add2(Two x, Two y) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(bits_of(x)), "l"(bits_of(y)));
  return two_of(d);
}
__device__ __forceinline__ Two exp2_approx(Two x) { return {exp2_approx(x.a), exp2_approx(x.b)}; }
__device__ __forceinline__ Two rcp_approx(Two x) { return {rcp_approx(x.a), rcp_approx(x.b)}; }
__device__ __forceinline__ Two at_most(Two x, float b) { return {at_most(x.a, b), at_most(x.b, b)}; }
__device__ __forceinline__ Two at_least(Two x, float b) { return {at_least(x.a, b), at_least(x.b, b)}; }

// e = exp(-x^2/2), and h with Phi(-x) = -e h, for x >= 0
__device__ __forceinline__ Two minus_tail(Two x, Two& e) {
  e = exp2_approx(mul2(mul2(x, x), both(-0.72134752f)));
  const Two t = rcp_approx(fma2(both(0.3f), x, both(1.0f)));
  Two p = both(-0.03542371094226837f);
  p = fma2(p, t, both(0.15615835785865784f));
  p = fma2(p, t, both(-0.2045566290616989f));
  p = fma2(p, t, both(0.05203389376401901f));
  p = fma2(p, t, both(-0.12769171595573425f));
  p = fma2(p, t, both(-0.10017596185207367f));
  p = fma2(p, t, both(-0.12071213126182556f));
  p = fma2(p, t, both(-0.11963200569152832f));
  return mul2(t, p);
}
__device__ __forceinline__ Two gelu_value(Two z) {  // z > 0: z (1 - Phi(-z))
  Two e;
  const Two x = at_most(Two{fabsf(z.a), fabsf(z.b)}, 64.0f), h = minus_tail(x, e);
  return fma2(mul2(x, e), h, Two{fmaxf(z.a, 0.0f), fmaxf(z.b, 0.0f)});
}
// With d = e (x phi(0) + h): 1 + d for z > 0 and -d for others, where the slope is small.  (1/2 added to what it is above 1/2, with z's sign, left no digit of slopes below
// 2^-24: at z = -4 1.5e-4 relative, at -5.5 all.)
__device__ __forceinline__ float one_above_zero(float z) {
  float y;
  asm("set.gt.f32.f32 %0, %1, 0f00000000;" : "=f"(y) : "f"(z));
  return y;
}
__device__ __forceinline__ Two gelu_slope(Two z) {
  Two e;
  const Two x = at_most(Two{fabsf(z.a), fabsf(z.b)}, 64.0f), h = minus_tail(x, e), one = {one_above_zero(z.a), one_above_zero(z.b)};
  return fma2(mul2(e, fma2(one, both(2.0f), both(-1.0f))), fma2(x, both(0.39894228f), h), one);
}
// z s(w) with w = z (one + cubic z^2): silu has one = 1, cubic = 0; gelu_tanh 2 sqrt(2/pi) (1, 0.044715)
struct Sigmoid {
  float one, cubic;
};
__device__ __forceinline__ Sigmoid sigmoid_of(int act) {
  return act == B2_ACT_SILU ? Sigmoid{1.0f, 0.0f} : Sigmoid{1.5957691216f, 0.0713548163f};
}
__device__ __forceinline__ Two sigmoid(Two w) { return rcp_approx(add2(both(1.0f), exp2_approx(mul2(w, both(-1.44269504f))))); }
__device__ __forceinline__ Two sigmoid_value(Two z, Sigmoid k) {
  const Two y = at_least(z, -64.0f), x = at_most(y, 64.0f);
  return mul2(y, sigmoid(mul2(x, fma2(mul2(x, x), both(k.cubic), both(k.one)))));
}
__device__ __forceinline__ Two sigmoid_slope(Two z, Sigmoid k) {
  const Two x = at_most(at_least(z, -64.0f), 64.0f), xx = mul2(x, x);
  const Two s = sigmoid(mul2(x, fma2(xx, both(k.cubic), both(k.one))));
  const Two rest = fma2(s, both(-1.0f), both(1.0f));
  return fma2(mul2(mul2(x, s), rest), fma2(xx, both(3.0f * k.cubic), both(k.one)), s);
}
__device__ __forceinline__ float relu_slope(float z) { return z > 0.0f ? 1.0f : z <= 0.0f ? 0.0f : z; }

// One test of the function for N numbers (even).
template <int N>
__device__ __forceinline__ void act_values(int act, float* v) {
  if (act == B2_ACT_RELU) {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = at_least(v[j], 0.0f);
  } else if (act == B2_ACT_GELU) {
#pragma unroll
    for (int j = 0; j < N; j += 2) {
      const Two y = gelu_value({v[j], v[j + 1]});
      v[j] = y.a, v[j + 1] = y.b;
    }
  } else if (act != B2_ACT_NONE) {
    const Sigmoid k = sigmoid_of(act);
#pragma unroll
    for (int j = 0; j < N; j += 2) {
      const Two y = sigmoid_value({v[j], v[j + 1]}, k);
      v[j] = y.a, v[j + 1] = y.b;
    }
  }
}
// v := v * act'(z)
template <int N>
__device__ __forceinline__ void act_slopes(int act, float* v, const float* z) {
  if (act == B2_ACT_RELU) {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] *= relu_slope(z[j]);
  } else if (act == B2_ACT_GELU) {
#pragma unroll
    for (int j = 0; j < N; j += 2) {
      const Two y = mul2({v[j], v[j + 1]}, gelu_slope({z[j], z[j + 1]}));
      v[j] = y.a, v[j + 1] = y.b;
    }
  } else if (act != B2_ACT_NONE) {
    const Sigmoid k = sigmoid_of(act);
#pragma unroll
    for (int j = 0; j < N; j += 2) {
      const Two y = mul2({v[j], v[j + 1]}, sigmoid_slope({z[j], z[j + 1]}, k));
      v[j] = y.a, v[j + 1] = y.b;
    }
  }
}

inline bool act_known(int act) { return act >= B2_ACT_NONE && act <= B2_ACT_SILU; }

}  // namespace b2
