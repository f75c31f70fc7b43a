// Block-scaled 8-bit numbers: e4m3 values with one scale for a block of 128, shared by the kernels that write and read
// them (b2_rmsnorm_f8, b2_quant_f8, b2_gemm_f8, b2_wgrad_f8).
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace b2 {

constexpr int kF8Block = 128;  // elements along the quantised (later summed) index that share a scale

// ---- the quantisation rule --------------------------------------------------------------------
// Largest magnitude as its bit pattern: for non-negative floats the integer order is the numeric order, and a NaN
// sorts above infinity, so that one integer maximum also says whether a block holds something that is not finite.
__device__ __forceinline__ uint32_t mag_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

constexpr uint32_t kScaleNan = 255;
// Scale byte of a block: the smallest 2^(b-127) with amax / 2^(b-127) <= 448 = 1.75 * 2^8.  Writing amax = f * 2^x with
// 1 <= f < 2 that power is x - 8, one more when f > 1.75 (mantissa field above 0x600000): integer arithmetic only.
__device__ __forceinline__ uint32_t f8_scale_byte(uint32_t amax_bits) {
  if (amax_bits >= 0x7f800000u) return kScaleNan;
  if (amax_bits == 0) return 127;
  const int b = (int)(amax_bits >> 23) - 8 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return (uint32_t)max(b, 0);
}
// 1 / scale, exact (b is at most 247 for a finite amax, so 254 - b is a normal exponent field).
__device__ __forceinline__ float f8_inv_scale(uint32_t b) { return __uint_as_float((254u - b) << 23); }

// four floats to four e4m3 numbers, the first in the lowest byte; round to nearest even
__device__ __forceinline__ uint32_t f8_pack4(float a, float b, float c, float d) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  return (uint32_t)lo | ((uint32_t)hi << 16);
}
// eight values of a block with the given scale byte
__device__ __forceinline__ uint2 f8_quant8(const float (&y)[8], uint32_t byte) {
  if (byte == kScaleNan) return make_uint2(0x7f7f7f7fu, 0x7f7f7f7fu);
  const float inv = f8_inv_scale(byte);
  return make_uint2(f8_pack4(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv),
                    f8_pack4(y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv));
}
// value of a scale byte (2^-127 is subnormal)
__device__ __forceinline__ float e8m0_value(uint32_t b) {
  return __uint_as_float(b == kScaleNan ? 0x7fc00000u : (b == 0 ? 0x00400000u : b << 23));
}

// ---- eight consecutive elements ----------------------------------------------------------------
// `vec`: the address is 16-byte aligned (uniform over a launch); nv of the eight exist (may be <= 0).
__device__ __forceinline__ void load8(const __nv_bfloat16* p, int64_t nv, bool vec, float (&v)[8]) {
  if (vec && nv >= 8) {
    const uint4 q = *reinterpret_cast<const uint4*>(p);
    const uint32_t u[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(u[i] << 16);
      v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < nv ? __bfloat162float(p[i]) : 0.0f;
  }
}
__device__ __forceinline__ void load8(const float* p, int64_t nv, bool vec, float (&v)[8]) {
  if (vec && nv >= 8) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < nv ? p[i] : 0.0f;
  }
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&p);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, int64_t nv, bool vec, const float (&v)[8]) {
  if (vec && nv >= 8) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < nv) p[i] = __float2bfloat16_rn(v[i]);
  }
}
__device__ __forceinline__ void store8(float* p, int64_t nv, bool vec, const float (&v)[8]) {
  if (vec && nv >= 8) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < nv) p[i] = v[i];
  }
}
// eight e4m3 numbers; `vec`: 8-byte aligned
__device__ __forceinline__ void store8_f8(uint8_t* p, int64_t nv, bool vec, uint2 q) {
  if (vec && nv >= 8) {
    *reinterpret_cast<uint2*>(p) = q;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < nv) p[i] = (uint8_t)((i < 4 ? q.x : q.y) >> (8 * (i & 3)));
  }
}

// columns of a matrix start on `bytes`-byte boundaries
inline bool columns_aligned(const void* p, int64_t ld, int elem, int bytes) {
  return (reinterpret_cast<uintptr_t>(p) % bytes) == 0 && ((uint64_t)ld * (uint64_t)elem) % (uint64_t)bytes == 0;
}

inline int64_t blocks_of(int64_t n, int64_t b) { return n / b + (n % b != 0); }

}  // namespace b2
