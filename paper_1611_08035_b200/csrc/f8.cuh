// Block-scaled 8-bit numbers: e4m3 values with one scale for a block of 128, shared by the kernels that write and read
// them (b2_rmsnorm_f8, b2_quant_f8, b2_gemm_f8, b2_wgrad_f8).
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "b2gemm.h"

namespace b2 {

// ---- launches that overlap the end of the kernel before ---------------------------------------------
// Every kernel of the 8-bit operators lets its successor in the stream be launched early (grid_started) and touches global memory
// only after its predecessor has completed and its writes are visible (grid_ready), so that setting up overlaps with finishing: a norm of
// eight tokens, called again and again, takes 3.4 us instead of 4.0.  Early is as soon as all CTAs run, or, in the products, as they come to their
// results: a successor's CTAs that come sooner take the places they find two to an SM (1001 x 999 x 1003: 10.3 us instead of 8.0).
// Kernels launched without the attribute are not affected.
__device__ __forceinline__ void grid_started() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void grid_ready() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
template <typename... Params, typename... Args>
inline int launch_overlapped_as(void (*kernel)(Params...), dim3 grid, unsigned threads, size_t smem, dim3 cluster, cudaStream_t st, const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid, cfg.blockDim = dim3(threads), cfg.dynamicSmemBytes = smem, cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim = {cluster.x, cluster.y, cluster.z};
  cfg.attrs = at, cfg.numAttrs = cluster.x * cluster.y * cluster.z > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, Params(args)...) == cudaSuccess ? B2_OK : B2_ERR_LAUNCH;
}
template <typename... Params, typename... Args>
inline int launch_overlapped(void (*kernel)(Params...), dim3 grid, unsigned threads, cudaStream_t st, const Args&... args) {
  return launch_overlapped_as(kernel, grid, threads, 0, dim3(1), st, args...);
}

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
// As they lie in memory.  Loading and unpacking are two steps so that several loads are on their way before the first is
// waited for: with the unpacking inside the load's branch, every load waited for the one before it (b2_quant_f8 of 16384 x
// 8192 bf16, eight numbers a load: 120 us instead of 84).
template <typename T>
struct Raw8 {
  uint32_t u[2 * sizeof(T)];
};
// `vec`: the address is 16-byte aligned (uniform over a launch); nv of the eight exist (may be <= 0), the others read as 0.
__device__ __forceinline__ void load8(const __nv_bfloat16* p, int64_t nv, bool vec, Raw8<__nv_bfloat16>& r) {
  if (vec && nv >= 8) {
    const uint4 q = *reinterpret_cast<const uint4*>(p);
    r.u[0] = q.x, r.u[1] = q.y, r.u[2] = q.z, r.u[3] = q.w;
  } else {
    const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      r.u[i] = (2 * i < nv ? (uint32_t)h[2 * i] : 0u) | ((2 * i + 1 < nv ? (uint32_t)h[2 * i + 1] : 0u) << 16);
  }
}
__device__ __forceinline__ void load8(const float* p, int64_t nv, bool vec, Raw8<float>& r) {
  const uint32_t* w = reinterpret_cast<const uint32_t*>(p);
  if (vec && nv >= 8) {
    const uint4 a = *reinterpret_cast<const uint4*>(w), b = *reinterpret_cast<const uint4*>(w + 4);
    r.u[0] = a.x, r.u[1] = a.y, r.u[2] = a.z, r.u[3] = a.w, r.u[4] = b.x, r.u[5] = b.y, r.u[6] = b.z, r.u[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) r.u[i] = i < nv ? w[i] : 0u;
  }
}
__device__ __forceinline__ void unpack8(const Raw8<__nv_bfloat16>& r, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(r.u[i] << 16);
    v[2 * i + 1] = __uint_as_float(r.u[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void unpack8(const Raw8<float>& r, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r.u[i]);
}
template <typename T>
__device__ __forceinline__ void load8(const T* p, int64_t nv, bool vec, float (&v)[8]) {
  Raw8<T> r;
  load8(p, nv, vec, r);
  unpack8(r, v);
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

// Eight numbers of a row for every lane of a warp that covers 256 consecutive ones starting at `first`.  VEC: every row
// starts on a 16-byte boundary and lane l holds numbers 8 l .. 8 l + 7, in whole loads; otherwise rows start anywhere and
// lane l holds l, l + 32, .., so that the lanes of every (narrow) load are neighbours (norm of 16384 x 1003 bf16: 50 us, 76 with narrow loads 16
// bytes apart).
template <typename T, bool VEC>
struct Warp256 {
  __device__ __forceinline__ static int index(int first, int j) {
    const int lane = threadIdx.x & 31;
    return VEC ? first + lane * 8 + j : first + j * 32 + lane;
  }
  __device__ __forceinline__ static void load(const T* row, int first, int n, Raw8<T>& r) {
    if constexpr (VEC) {
      load8(row + index(first, 0), n - index(first, 0), true, r);
    } else if constexpr (sizeof(T) == 2) {
      const uint16_t* h = reinterpret_cast<const uint16_t*>(row);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int a = index(first, 2 * j), b = index(first, 2 * j + 1);
        r.u[j] = (a < n ? (uint32_t)h[a] : 0u) | (b < n ? (uint32_t)h[b] : 0u) << 16;
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) r.u[j] = index(first, j) < n ? reinterpret_cast<const uint32_t*>(row)[index(first, j)] : 0u;
    }
  }
  __device__ __forceinline__ static void store(T* row, int first, int n, const float (&v)[8]) {
    if constexpr (VEC) {
      store8(row + index(first, 0), n - index(first, 0), true, v);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (index(first, j) < n) {
          if constexpr (sizeof(T) == 2) row[index(first, j)] = __float2bfloat16_rn(v[j]);
          else row[index(first, j)] = v[j];
        }
    }
  }
  // Quantise the two blocks of 128 and write them with their scales; numbers beyond the row are 0.
  __device__ __forceinline__ static void quantise(const float (&y)[8], uint8_t* q, uint8_t* s, int first, int n) {
    const int lane = threadIdx.x & 31;
    if constexpr (VEC) {
      uint32_t m = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) m = max(m, mag_bits(y[j]));
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
      const uint32_t byte = f8_scale_byte(m);
      const int e = index(first, 0);
      if (e < n) {
        store8_f8(q + e, n - e, true, f8_quant8(y, byte));
        if ((lane & 15) == 0) s[e / kF8Block] = (uint8_t)byte;
      }
    } else {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) m = max(m, mag_bits(y[4 * b + j]));
        const uint32_t byte = f8_scale_byte(__reduce_max_sync(0xffffffffu, m));
        const float inv = byte == kScaleNan ? 0.0f : f8_inv_scale(byte);
        const uint32_t w = byte == kScaleNan ? 0x7f7f7f7fu : f8_pack4(y[4 * b] * inv, y[4 * b + 1] * inv, y[4 * b + 2] * inv, y[4 * b + 3] * inv);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (index(first, 4 * b + j) < n) q[index(first, 4 * b + j)] = (uint8_t)(w >> (8 * j));
        if (lane == 0 && first + 128 * b < n) s[first / kF8Block + b] = (uint8_t)byte;
      }
    }
  }
};

// columns of a matrix start on `bytes`-byte boundaries
inline bool columns_aligned(const void* p, int64_t ld, int elem, int bytes) {
  return (reinterpret_cast<uintptr_t>(p) % bytes) == 0 && ((uint64_t)ld * (uint64_t)elem) % (uint64_t)bytes == 0;
}

// Quotient of 32-bit numbers by one fixed divisor: a multiplication and a shift.  With 2^(l-1) < d <= 2^l and
// mul = floor(2^32 (2^l - d) / d) + 1, n / d = (mulhi(mul, n) + n) >> l exactly (the sum taken in 33 bits).
struct FastDiv {
  uint32_t d, mul, shift;
};
inline FastDiv fast_div(uint32_t d) {
  uint32_t l = 0;
  while (l < 32 && (1ull << l) < d) ++l;
  return {d, (uint32_t)((((1ull << l) - d) << 32) / d + 1), l};
}
__device__ __forceinline__ uint32_t div_by(uint32_t n, const FastDiv& f) {
  return (uint32_t)(((uint64_t)__umulhi(f.mul, n) + n) >> f.shift);
}

constexpr int64_t kMostFeatures = 0x7fffffffLL - 8192;  // positions in a token are 32-bit numbers

inline int64_t blocks_of(int64_t n, int64_t b) { return n / b + (n % b != 0); }

}  // namespace b2
