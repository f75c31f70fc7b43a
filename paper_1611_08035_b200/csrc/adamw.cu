// One AdamW step over all tensors of a list, moments in fp32 or in 8 bits.
//
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,  p = p (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v / (1 - b2^t)) + eps)
//
// Bound by memory: 14 bytes an element with fp32 parameters, bf16 gradients and states in 8 bits, 28 with everything in fp32.  The list travels as a kernel
// argument; a CTA finds its tensor by bisection among the tensors' first CTAs.  A warp holds whole blocks of 128 of an 8-bit state, whose largest magnitudes never leave it.
// Measured: 268 million parameters in 8 bits 659 us (5.7 TB/s, 87 % of the copy rate), 716 after a tenth of a second, when the board's power limit takes the clock to 1.7 GHz; 25
// million in fp32 that start anywhere 119 us (5.9 TB/s); ten tensors of 790 thousand elements 4.7 us.
//
// States in 8 bits: m and r = sqrt(v) (half the exponent range of v, which e4m3's seventeen binades are then enough for) are rounded at random, so that the mean over
// steps is right although a step moves r by less than half the distance of two e4m3 numbers.  The twenty random bits come from the element's number, a hash for
// eight elements and an addition for each.  m and v are computed by single roundings in a fixed order (no fused multiply-adds), and so is r: then everyone who
// computes them in fp32 comes to the same bits, and to the same side of a random rounding.
#include <algorithm>

#include "act.cuh"
#include "b2gemm.h"
#include "common.cuh"
#include "entry.h"
#include "f8.cuh"

namespace b2 {
namespace {

struct AdamTensor {
  void* p;
  const void* g;
  void *m, *v;
  uint8_t *sm, *sv;
  int64_t n;
  uint64_t first;  // number of the first element, through the list
  int vec;         // all pointers are aligned for whole loads
};
template <int MOST>
struct AdamList {
  int count;
  uint32_t cta[MOST];  // first CTA of each tensor
  AdamTensor t[MOST];
};
struct AdamStep {
  float b1, a1, b2, a2, eps;   // a = 1 - b
  float decay, size, root;     // 1 - lr wd, lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
  uint32_t key;
  uint64_t seed;
  const float *scale, *lr_device;
  const int64_t* step_device;
  double lr, wd, log_b1, log_b2;
  int64_t step;
};
// A warp has PIECES times 256 elements: two, or one where the list is too short to give every SM several CTAs of that (ten tensors of 790 thousand elements 7.7 us on the GPU with two,
// 4.7 with one).
__host__ __device__ constexpr int unit(int pieces) { return 8 * 256 * pieces; }  // elements of a CTA

// The finaliser of MurmurHash3 (Austin Appleby, public domain).
__host__ __device__ __forceinline__ uint32_t fmix(uint32_t x) {
  x = (x ^ (x >> 16)) * 0x85EBCA6Bu;
  x = (x ^ (x >> 13)) * 0xC2B2AE35u;
  return x ^ (x >> 16);
}
constexpr uint32_t kGolden = 0x9E3779B9u;
__host__ __device__ __forceinline__ uint32_t adam_key(uint64_t seed, int64_t step) {
  return fmix(fmix(fmix((uint32_t)seed) ^ (uint32_t)(seed >> 32)) ^ (uint32_t)step);
}
// What depends on the step's number and the learning rate.
__host__ __device__ __forceinline__ void adam_factors(AdamStep& s, double lr, int64_t step) {
  s.decay = (float)(1.0 - lr * s.wd);
  s.size = (float)(lr / -expm1((double)step * s.log_b1));
  s.root = (float)(1.0 / sqrt(-expm1((double)step * s.log_b2)));
  s.key = adam_key(s.seed, step);
}

// Four e4m3 numbers of a word.
__device__ __forceinline__ void f8_unpack4(uint32_t w, float* v) {
  uint32_t lo, hi;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(lo) : "h"((uint16_t)w));
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(hi) : "h"((uint16_t)(w >> 16)));
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(v[0]), "=f"(v[1]) : "r"(lo));
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(v[2]), "=f"(v[3]) : "r"(hi));
}
// y, |y| <= 448, to a neighbouring e4m3 number: with 20 random bits added below the third place of the mantissa, the rest is cut.  Numbers below 2^-6 have
// one distance, 2^-9, as those of the binade from 2^-6 on have, where they are taken for it.
__device__ __forceinline__ float f8_at_random(float y, uint32_t bits20) {
  const bool small = fabsf(y) < 0.015625f;
  const float c = __uint_as_float((__float_as_uint(y) & 0x80000000u) | 0x3c800000u);  // 2^-6 with y's sign
  float t = small ? __fadd_rn(y, c) : y;
  t = __uint_as_float((__float_as_uint(t) + bits20) & 0xfff00000u);
  return small ? __fadd_rn(t, -c) : t;
}

// m, v and p of one element, in place; r = sqrt(v).
template <bool ROOT_GIVEN>
__device__ __forceinline__ void adam_element(const AdamStep& s, float g, float& p, float& m, float& v, float& r) {
  if (ROOT_GIVEN) v = __fmul_rn(r, r);
  m = __fadd_rn(__fmul_rn(m, s.b1), __fmul_rn(g, s.a1));
  v = __fadd_rn(__fmul_rn(v, s.b2), __fmul_rn(__fmul_rn(g, g), s.a2));
  r = __fsqrt_rn(v);
  p = __fadd_rn(__fmul_rn(p, s.decay), -__fdividef(s.size * m, fmaf(r, s.root, s.eps)));
}

template <typename TP, typename TG, int BITS, bool VEC, int PIECES>
__device__ __forceinline__ void adam_pieces(const AdamTensor& t, const AdamStep& s, float scale, int64_t at0) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t at = at0 + warp * 256 * PIECES;
  if (at >= t.n) return;
  const int n = (int)min((int64_t)(256 * PIECES), t.n - at);  // elements of this warp
  TP* P = static_cast<TP*>(t.p) + at;
  const TG* G = static_cast<const TG*>(t.g) + at;
  using AtP = Warp256<TP, VEC>;
  using AtG = Warp256<TG, VEC>;
  using At4 = Warp256<float, VEC>;
  Raw8<TP> p8[PIECES];
  Raw8<TG> g8[PIECES];
#pragma unroll
  for (int u = 0; u < PIECES; ++u) {
    AtP::load(P, 256 * u, n, p8[u]);
    AtG::load(G, 256 * u, n, g8[u]);
  }
  if constexpr (BITS == 32) {
    float *M = static_cast<float*>(t.m) + at, *V = static_cast<float*>(t.v) + at;
    Raw8<float> m8[PIECES], v8[PIECES];
#pragma unroll
    for (int u = 0; u < PIECES; ++u) {
      At4::load(M, 256 * u, n, m8[u]);
      At4::load(V, 256 * u, n, v8[u]);
    }
#pragma unroll
    for (int u = 0; u < PIECES; ++u) {
      float p[8], g[8], m[8], v[8], r;
      unpack8(p8[u], p), unpack8(g8[u], g), unpack8(m8[u], m), unpack8(v8[u], v);
#pragma unroll
      for (int j = 0; j < 8; ++j) adam_element<false>(s, __fmul_rn(g[j], scale), p[j], m[j], v[j], r);
      AtP::store(P, 256 * u, n, p);
      At4::store(M, 256 * u, n, m);
      At4::store(V, 256 * u, n, v);
    }
  } else {
    static_assert(!VEC, "aligned elements are adam_aligned's");
    uint8_t *M = static_cast<uint8_t*>(t.m) + at, *R = static_cast<uint8_t*>(t.v) + at;
    uint8_t *SM = t.sm + at / kF8Block, *SR = t.sv + at / kF8Block;
    uint32_t m8[PIECES][2], r8[PIECES][2], sm[PIECES][2], sr[PIECES][2];  // half h of a lane's numbers is of block h
#pragma unroll
    for (int u = 0; u < PIECES; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        m8[u][h] = r8[u][h] = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int e = 256 * u + 128 * h + 32 * j + lane;
          if (e < n) m8[u][h] |= (uint32_t)M[e] << (8 * j), r8[u][h] |= (uint32_t)R[e] << (8 * j);
        }
        const int b = 2 * u + h;
        sm[u][h] = b * kF8Block < n ? SM[b] : 127u, sr[u][h] = b * kF8Block < n ? SR[b] : 127u;
      }
    const uint64_t e0 = t.first + (uint64_t)at;
#pragma unroll
    for (int u = 0; u < PIECES; ++u) {
      float p[8], g[8], m[8], r[8];
      unpack8(p8[u], p), unpack8(g8[u], g);
      f8_unpack4(m8[u][0], m), f8_unpack4(m8[u][1], m + 4), f8_unpack4(r8[u][0], r), f8_unpack4(r8[u][1], r + 4);
      uint32_t most_m[2] = {0, 0}, most_r[2] = {0, 0};
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float v;
        m[j] = __fmul_rn(m[j], e8m0_value(sm[u][j >> 2])), r[j] = __fmul_rn(r[j], e8m0_value(sr[u][j >> 2]));
        adam_element<true>(s, __fmul_rn(g[j], scale), p[j], m[j], v, r[j]);
        most_m[j >> 2] = max(most_m[j >> 2], mag_bits(m[j])), most_r[j >> 2] = max(most_r[j >> 2], mag_bits(r[j]));
      }
      AtP::store(P, 256 * u, n, p);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t byte_m = f8_scale_byte(__reduce_max_sync(0xffffffffu, most_m[h])), byte_r = f8_scale_byte(__reduce_max_sync(0xffffffffu, most_r[h]));
        const float inv_m = byte_m == kScaleNan ? 0.0f : f8_inv_scale(byte_m), inv_r = byte_r == kScaleNan ? 0.0f : f8_inv_scale(byte_r);
        float a[4], b[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint64_t e = e0 + 256 * u + 128 * h + 32 * j + lane, e8 = e >> 3;
          const uint32_t hm = fmix((uint32_t)e8 + fmix((uint32_t)(e8 >> 32) + s.key)), hr = fmix(hm + kGolden), i = ((uint32_t)e & 7u) * kGolden;
          a[j] = f8_at_random(__fmul_rn(m[4 * h + j], inv_m), (hm + i) >> 12);
          const float y = __fmul_rn(r[4 * h + j], inv_r);
          b[j] = f8_at_random(y, (hr + i) >> 12);
          b[j] = y > 0.0f ? fmaxf(b[j], 0.001953125f) : b[j];  // 2^-9
        }
        const uint32_t qm = byte_m == kScaleNan ? 0x7f7f7f7fu : f8_pack4(a[0], a[1], a[2], a[3]);
        const uint32_t qr = byte_r == kScaleNan ? 0x7f7f7f7fu : f8_pack4(b[0], b[1], b[2], b[3]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int e = 256 * u + 128 * h + 32 * j + lane;
          if (e < n) M[e] = (uint8_t)(qm >> (8 * j)), R[e] = (uint8_t)(qr >> (8 * j));
        }
        if (lane == 0 && 256 * u + 128 * h < n) SM[2 * u + h] = (uint8_t)byte_m, SR[2 * u + h] = (uint8_t)byte_r;
      }
    }
  }
}

// ---- 512 or 256 aligned elements of a warp, states in 8 bits -----------------------------------------------------------------
// 14 bytes an element leave a GPU some eighty instructions for it, which one at a time they were not enough (109: 1000 us for 268 million elements, 574 by the bytes).  So this
// path does as much as it can two numbers at a time and gives a lane sixteen (or eight) consecutive elements, eight (or sixteen) lanes to a block.  Numbers below 2^-6 of their scale, whose
// distance is not the binade's, take a branch; a warp with a v for which the root below is not exact, or not finite, goes to adam_pieces before it has written anything.

// A sum of products that are rounded before: the packed addition is joined with them to a multiply-add (4 of 16 million first moments fell to the other side of their rounding).
__device__ __forceinline__ Two sum_rn(Two x, Two y) { return {__fadd_rn(x.a, y.a), __fadd_rn(x.b, y.b)}; }
// Minus the square roots of -n, n <= 0, rounded to nearest: an approximation of the reciprocal root, and from it one Newton step on the root with the exact remainder (P.
// Markstein, IBM Journal of Research and Development 34, 1990); all signs turned, so that none is in the way of the packed instructions.  0, and 2^-100 to the largest finite
// number, give __fsqrt_rn's results: compared once on the GPU, every mantissa with the exponents 0, -2, 20, 98, -50 and -100 and the next ones.
__device__ __forceinline__ float rsqrt_approx(float x) {
  float y;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ Two minus_sqrt2_rn(Two n) {
  const Two y = {rsqrt_approx(fmaxf(-n.a, 0x1p-100f)), rsqrt_approx(fmaxf(-n.b, 0x1p-100f))}, s = mul2(n, y), h = mul2(y, both(0.5f));
  return fma2(fma2(s, s, n), h, s);
}
// of three magnitudes
__device__ __forceinline__ float largest_nan(float a, float b, float c) {
  float y;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
__device__ __forceinline__ float smallest(float a, float b, float c) {
  float y;
  asm("min.abs.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
// E magnitudes' largest, NaN where there is one, and smallest.
struct Extent {
  float most, least;
};
template <int E>
__device__ __forceinline__ Extent extent_of(const float* x) {
  Extent e{fabsf(x[0]), fabsf(x[0])};
#pragma unroll
  for (int j = 1; j + 1 < E; j += 2) e.most = largest_nan(e.most, x[j], x[j + 1]), e.least = smallest(e.least, x[j], x[j + 1]);
  return {largest_nan(e.most, x[E - 1], x[E - 1]), smallest(e.least, x[E - 1], x[E - 1])};
}
// E numbers of a block as e4m3, with the random bits of a hash for each eight of them.  ROOT: they are the roots' negatives.
template <bool ROOT, int E>
__device__ __forceinline__ void quantise_at_random(const float* x, uint32_t byte, float least, const uint32_t (&h)[2], uint32_t (&w)[E / 4]) {
  if (byte == kScaleNan) {
#pragma unroll
    for (int i = 0; i < E / 4; ++i) w[i] = 0x7f7f7f7fu;
    return;
  }
  const float inv = ROOT ? -f8_inv_scale(byte) : f8_inv_scale(byte);
  const bool plain = least * fabsf(inv) >= 0.015625f;
#pragma unroll
  for (int i = 0; i < E / 4; ++i) {
    float t[4];
#pragma unroll
    for (int j = 0; j < 4; j += 2) {
      const Two y = mul2({x[4 * i + j], x[4 * i + j + 1]}, both(inv));
      t[j] = y.a, t[j + 1] = y.b;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t bits = (h[i / 2] + (uint32_t)((4 * i + j) & 7) * kGolden) >> 12;
      if (plain) {
        t[j] = __uint_as_float((__float_as_uint(t[j]) + bits) & 0xfff00000u);
      } else {
        const float y = t[j];
        t[j] = f8_at_random(y, bits);
        if (ROOT) t[j] = y > 0.0f ? fmaxf(t[j], 0.001953125f) : t[j];
      }
    }
    w[i] = f8_pack4(t[0], t[1], t[2], t[3]);
  }
}
// 4 Q bytes of a lane as they lie in memory, aligned to 16
template <int Q>
__device__ __forceinline__ void load_words(const void* p, uint32_t (&w)[Q]) {
#pragma unroll
  for (int i = 0; i < Q / 4; ++i) {
    const uint4 q = static_cast<const uint4*>(p)[i];
    w[4 * i] = q.x, w[4 * i + 1] = q.y, w[4 * i + 2] = q.z, w[4 * i + 3] = q.w;
  }
}
template <typename T, int Q>
__device__ __forceinline__ Two pair_at(const uint32_t (&w)[Q], int i) {
  if constexpr (sizeof(T) == 2) return {__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u)};
  else return {__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1])};
}
template <typename T, int E>
__device__ __forceinline__ void store_numbers(T* p, const float* v) {
#pragma unroll
  for (int i = 0; i < E; i += 8) {
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = v[i + j];
    store8(p + i, 8, true, x);
  }
}
// E bytes, aligned to 8
template <int E>
__device__ __forceinline__ void load_bytes(const uint8_t* p, uint32_t (&w)[E / 4]) {
#pragma unroll
  for (int i = 0; i < E / 8; ++i) {
    const uint2 a = reinterpret_cast<const uint2*>(p)[i];
    w[2 * i] = a.x, w[2 * i + 1] = a.y;
  }
}
template <int E>
__device__ __forceinline__ void store_bytes(uint8_t* p, const uint32_t (&w)[E / 4]) {
#pragma unroll
  for (int i = 0; i < E / 8; ++i) reinterpret_cast<uint2*>(p)[i] = make_uint2(w[2 * i], w[2 * i + 1]);
}

// False, with nothing written, where a root is not exact.
template <typename TP, typename TG, int E>
__device__ __forceinline__ bool adam_aligned(const AdamTensor& t, const AdamStep& s, float scale, int64_t at) {
  constexpr int L = kF8Block / E;  // lanes of a block
  const int lane = threadIdx.x & 31, block = lane / L;
  const int64_t e0 = at + E * lane;
  TP* P = static_cast<TP*>(t.p) + e0;
  uint8_t *M = static_cast<uint8_t*>(t.m) + e0, *R = static_cast<uint8_t*>(t.v) + e0, *SM = t.sm + at / kF8Block + block, *SR = t.sv + at / kF8Block + block;
  uint32_t pq[E * sizeof(TP) / 4], gq[E * sizeof(TG) / 4], mq[E / 4], rq[E / 4];
  load_words(P, pq);
  load_words(static_cast<const TG*>(t.g) + e0, gq);
  load_bytes<E>(M, mq), load_bytes<E>(R, rq);
  const float sm = e8m0_value(*SM), sr = e8m0_value(*SR);
  float p[E], m[E], r[E];  // r: minus the root
#pragma unroll
  for (int i = 0; i < E / 4; ++i) {
    float a[4], b[4];
    f8_unpack4(mq[i], a), f8_unpack4(rq[i], b);
#pragma unroll
    for (int j = 0; j < 4; j += 2) {
      const int k = 4 * i + j;
      const Two g = mul2(pair_at<TG>(gq, k / 2), both(scale));
      const Two mo = mul2({a[j], a[j + 1]}, both(sm)), ro = mul2({b[j], b[j + 1]}, both(sr));
      const Two mn = sum_rn(mul2(mo, both(s.b1)), mul2(g, both(s.a1)));
      const Two minus_v = sum_rn(mul2(mul2(ro, ro), both(-s.b2)), mul2(mul2(g, g), both(-s.a2)));
      const Two rn = minus_sqrt2_rn(minus_v);
      const Two inv = rcp_approx(fma2(rn, both(-s.root), both(s.eps)));
      const Two pn = fma2(mul2(mn, both(-s.size)), inv, mul2(pair_at<TP>(pq, k / 2), both(s.decay)));
      m[k] = mn.a, m[k + 1] = mn.b, r[k] = rn.a, r[k + 1] = rn.b, p[k] = pn.a, p[k + 1] = pn.b;
    }
  }
  const Extent em = extent_of<E>(m), er = extent_of<E>(r);
  bool exact = er.most <= 0x1p64f;  // not NaN
  if (er.least < 0x1p-50f) {
#pragma unroll
    for (int k = 0; k < E; ++k) exact = exact && (r[k] == 0.0f || r[k] <= -0x1p-50f);
  }
  if (!__all_sync(0xffffffffu, exact)) return false;
  store_numbers<TP, E>(P, p);
  float am = em.most, ar = er.most;
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) am = larger_nan(am, __shfl_xor_sync(0xffffffffu, am, o)), ar = larger_nan(ar, __shfl_xor_sync(0xffffffffu, ar, o));
  const uint32_t bm = f8_scale_byte(__float_as_uint(am)), br = f8_scale_byte(__float_as_uint(ar));
  const uint64_t e8 = (t.first + (uint64_t)e0) >> 3;  // even where there are two hashes: both have the same high half
  const uint32_t high = fmix((uint32_t)(e8 >> 32) + s.key);
  uint32_t h[2], g[2], w[E / 4];
#pragma unroll
  for (int i = 0; i < 2; ++i) h[i] = fmix((uint32_t)e8 + (uint32_t)i + high), g[i] = fmix(h[i] + kGolden);
  quantise_at_random<false, E>(m, bm, em.least, h, w);
  store_bytes<E>(M, w);
  quantise_at_random<true, E>(r, br, er.least, g, w);
  store_bytes<E>(R, w);
  if (lane % L == 0) *SM = (uint8_t)bm, *SR = (uint8_t)br;
  return true;
}

template <typename TP, typename TG, int BITS, int MOST, int PIECES>
__global__ void __launch_bounds__(256, BITS == 8 ? 3 : 2) adamw_kernel(const __grid_constant__ AdamList<MOST> list, AdamStep s) {
  grid_started();
  int lo = 0, hi = list.count;  // the last tensor whose first CTA is not after this one
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (list.cta[mid] <= blockIdx.x) lo = mid;
    else hi = mid;
  }
  const AdamTensor& t = list.t[lo];
  grid_ready();
  if (s.step_device || s.lr_device) adam_factors(s, s.lr_device ? (double)*s.lr_device : s.lr, s.step_device ? *s.step_device : s.step);
  const float scale = s.scale ? *s.scale : 1.0f;
  const int64_t at = (int64_t)(blockIdx.x - list.cta[lo]) * unit(PIECES);
  if constexpr (BITS == 8) {
    const int64_t mine = at + (threadIdx.x >> 5) * (256 * PIECES);
    if (t.vec && mine + 256 * PIECES <= t.n && adam_aligned<TP, TG, 8 * PIECES>(t, s, scale, mine)) return;
    adam_pieces<TP, TG, 8, false, PIECES>(t, s, scale, at);  // also what does not start on 16 bytes, and the ends
  } else {
    if (t.vec) adam_pieces<TP, TG, 32, true, PIECES>(t, s, scale, at);
    else adam_pieces<TP, TG, 32, false, PIECES>(t, s, scale, at);
  }
}

template <typename TP, typename TG, int BITS, int PIECES, int MOST>
int adam_launch(const AdamList<MOST>& list, unsigned ctas, const AdamStep& s, cudaStream_t st) {
  return launch_overlapped(adamw_kernel<TP, TG, BITS, MOST, PIECES>, ctas, 256, st, list, s);
}
template <int PIECES, int MOST>
int adam_launch_kind(int kind, const AdamList<MOST>& list, unsigned ctas, const AdamStep& s, cudaStream_t st) {
  using F = float;
  using B = __nv_bfloat16;
  switch (kind) {
    case 0: return adam_launch<F, F, 32, PIECES>(list, ctas, s, st);
    case 1: return adam_launch<F, B, 32, PIECES>(list, ctas, s, st);
    case 2: return adam_launch<B, F, 32, PIECES>(list, ctas, s, st);
    case 3: return adam_launch<B, B, 32, PIECES>(list, ctas, s, st);
    case 4: return adam_launch<F, F, 8, PIECES>(list, ctas, s, st);
    case 5: return adam_launch<F, B, 8, PIECES>(list, ctas, s, st);
    case 6: return adam_launch<B, F, 8, PIECES>(list, ctas, s, st);
    default: return adam_launch<B, B, 8, PIECES>(list, ctas, s, st);
  }
}

bool aligned(const void* p, int to) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)to == 0; }
bool adam_valid(const b2_adamw_tensor& t) {
  if (t.n < 0 || t.reserved != 0 || (t.state_bits != 8 && t.state_bits != 32)) return false;
  if ((t.type_param != B2_TYPE_F32 && t.type_param != B2_TYPE_BF16) || (t.type_grad != B2_TYPE_F32 && t.type_grad != B2_TYPE_BF16)) return false;
  if (t.n == 0) return true;
  if (!t.param || !t.grad || !t.m || !t.v || (t.state_bits == 8 && (!t.sm || !t.sv))) return false;
  const int states = t.state_bits == 8 ? 1 : 4;
  return aligned(t.param, t.type_param == B2_TYPE_BF16 ? 2 : 4) && aligned(t.grad, t.type_grad == B2_TYPE_BF16 ? 2 : 4) && aligned(t.m, states) && aligned(t.v, states);
}
// Whether no parameter shares memory with another: a tensor that occurs twice would be updated by two CTAs at once.  2048 ranges at a time, sorted, on the stack: no call allocates.
struct AdamRange {
  uintptr_t begin, end;
};
constexpr int kRanges = 2048;
int adam_ranges(const b2_adamw_tensor* tensors, int count, AdamRange* r) {
  int n = 0;
  for (int i = 0; i < count && i < kRanges; ++i) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(tensors[i].param);
    if (tensors[i].n > 0) r[n++] = {at, at + (uintptr_t)tensors[i].n * (tensors[i].type_param == B2_TYPE_BF16 ? 2 : 4)};
  }
  std::sort(r, r + n, [](const AdamRange& a, const AdamRange& b) { return a.begin < b.begin; });
  return n;
}
bool adam_apart(const b2_adamw_tensor* tensors, int count) {
  AdamRange a[kRanges], b[kRanges];
  for (int64_t i = 0; i < count; i += kRanges) {
    const int na = adam_ranges(tensors + i, count - (int)i, a);
    for (int k = 1; k < na; ++k)
      if (a[k].begin < a[k - 1].end) return false;
    for (int64_t j = i + kRanges; j < count; j += kRanges) {
      const int nb = adam_ranges(tensors + j, count - (int)j, b);
      for (int x = 0, y = 0; x < na && y < nb;) {
        if (a[x].begin < b[y].end && b[y].begin < a[x].end) return false;
        if (a[x].end <= b[y].begin) ++x;
        else ++y;
      }
    }
  }
  return true;
}
int adam_kind(const b2_adamw_tensor& t) { return (t.state_bits == 8 ? 4 : 0) + (t.type_param == B2_TYPE_BF16 ? 2 : 0) + (t.type_grad == B2_TYPE_BF16 ? 1 : 0); }

// The tensors of one kind, MOST at a time.
template <int PIECES, int MOST>
int adam_run(const b2_adamw_tensor* tensors, int count, int kind, const AdamStep& s, cudaStream_t st) {
  AdamList<MOST> list;
  list.count = 0;
  int64_t ctas = 0;
  uint64_t first = 0;
  auto flush = [&]() {
    const int rc = list.count ? adam_launch_kind<PIECES>(kind, list, (unsigned)ctas, s, st) : B2_OK;
    list.count = 0, ctas = 0;
    return rc;
  };
  for (int i = 0; i < count; ++i) {
    const b2_adamw_tensor& t = tensors[i];
    if (t.n > 0 && adam_kind(t) == kind) {
      const int64_t more = blocks_of(t.n, unit(PIECES));
      if (list.count == MOST || ctas + more > 0x7fffffffLL) {
        const int rc = flush();
        if (rc) return rc;
      }
      const int states = t.state_bits == 8 ? 8 : 16;
      const bool vec = aligned(t.param, 16) && aligned(t.grad, 16) && aligned(t.m, states) && aligned(t.v, states);
      list.cta[list.count] = (uint32_t)ctas;
      list.t[list.count++] = {t.param, t.grad, t.m, t.v, static_cast<uint8_t*>(t.sm), static_cast<uint8_t*>(t.sv), t.n, first, vec};
      ctas += more;
    }
    first += (uint64_t)blocks_of(t.n, kF8Block) * kF8Block;
  }
  return flush();
}

}  // namespace
}  // namespace b2

extern "C" int b2_adamw(const b2_adamw_tensor* tensors, int count, double lr, double beta1, double beta2, double eps, double weight_decay,
                        int64_t step, uint64_t seed, const float* grad_scale, const float* lr_device, const int64_t* step_device,
                        void* cuda_stream) {
  using namespace b2;
  if (count > 0 && !tensors) return -1;
  if (count < 0) return -2;
  if (!lr_device && !(lr - lr == 0.0)) return -3;  // infinite or NaN
  if (!(beta1 >= 0.0 && beta1 < 1.0)) return -4;
  if (!(beta2 >= 0.0 && beta2 < 1.0)) return -5;
  if (!(eps >= 0.0)) return -6;
  if (!(weight_decay - weight_decay == 0.0)) return -7;
  if (!step_device && step < 1) return -8;
  int of_kind[8] = {};
  double elements[8] = {};
  for (int i = 0; i < count; ++i) {
    if (!adam_valid(tensors[i]) || blocks_of(tensors[i].n, unit(1)) > 0x7fffffffLL) return -1;
    if (tensors[i].n > 0) ++of_kind[adam_kind(tensors[i])], elements[adam_kind(tensors[i])] += (double)tensors[i].n;
  }
  if (!adam_apart(tensors, count)) return -1;
  AdamStep s = {};
  s.b1 = (float)beta1, s.a1 = (float)(1.0 - beta1), s.b2 = (float)beta2, s.a2 = (float)(1.0 - beta2), s.eps = (float)eps;
  s.seed = seed, s.scale = grad_scale, s.lr_device = lr_device, s.step_device = step_device;
  s.lr = lr, s.wd = weight_decay, s.log_b1 = log(beta1), s.log_b2 = log(beta2), s.step = step;
  if (!lr_device && !step_device) adam_factors(s, lr, step);
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  for (int kind = 0; kind < 8; ++kind) {
    if (of_kind[kind] == 0) continue;
    const bool few = of_kind[kind] <= 12, small = elements[kind] < (double)unit(2) * 3 * sm_count_cached();
    const int rc = !few ? adam_run<2, 240>(tensors, count, kind, s, st) : small ? adam_run<1, 12>(tensors, count, kind, s, st) : adam_run<2, 12>(tensors, count, kind, s, st);
    if (rc) return rc;
  }
  return B2_OK;
}
