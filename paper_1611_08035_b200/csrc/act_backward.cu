// The backward pass of an activation and a bias:
//
//   dz = dy act'(z),   db_i = sum over tokens of dz_i,   (q, s) = dz quantised in blocks of 128 features of a token
//
// Bound by memory: dy and z are read once, dz and q written once.  The eight warps of a CTA take the same features of different tokens, so that a feature's sum
// stays in one lane's register over all of a warp's tokens; what is left to add are eight numbers a CTA and one a CTA of the same features, in a fixed order.  A lane has 16
// or 32 bytes of a token and does two numbers an instruction; two more tokens are on their way while it works on one.
// Measured, tokens x features: 8192 x 16384 bf16 with z, dz, q and db 172 us (5.5 TB/s, 83 % of the copy rate; what is left is instructions, two of them of the unit for
// exp and 1/x, an element); 8192 x 4096 without z or dz 18-24 us (of 15); 33 x 1003 fp32 3.3 us in a captured graph.
#include "act.cuh"
#include "b2gemm.h"
#include "common.cuh"
#include "entry.h"
#include "f8.cuh"

namespace b2 {
namespace {

struct ActBwdArgs {
  int d, act;
  int64_t t, per;  // tokens; tokens of a CTA
  const void *DY, *Z;
  void *DZ, *Q, *S;
  int64_t lddy, ldz, lddz, ldq, lds;
  float* sums;  // [gridDim.y][d], or db itself
};
constexpr int kTokens = 2;  // of a warp at a time, where columns start anywhere
constexpr int kMostCluster = 8;

// A CTA's sums of `width` features from `first` on, one row of `part` a warp: to p.sums, or, CL, added over the cluster's CTAs first, in the order of their rank.
template <bool CL>
__device__ __forceinline__ void act_sum_up(const ActBwdArgs& p, float* part, int width, int first) {
  __syncthreads();
  for (int i = threadIdx.x; i < width; i += 256) {
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < 8; ++w) s += part[w * width + i];
    if (CL) part[i] = s;  // the same thread's column
    else if (first + i < p.d) p.sums[blockIdx.y * (int64_t)p.d + first + i] = s;
  }
  if constexpr (CL) {
    cluster_sync_all();
    if (blockIdx.y == 0) {
      for (int i = threadIdx.x; i < width; i += 256) {
        float s = 0.0f, x[kMostCluster];
#pragma unroll
        for (int q = 0; q < kMostCluster; ++q) {
          x[q] = 0.0f;
          if (q < (int)gridDim.y) asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x[q]) : "r"(cluster_map_shared(smem_u32(part + i), (uint32_t)q)));
        }
#pragma unroll
        for (int q = 0; q < kMostCluster; ++q) s += x[q];
        if (first + i < p.d) p.sums[first + i] = s;
      }
    }
    cluster_sync_all();  // no CTA leaves before its sums have been read
  }
}

// 16 Q bytes of a row, aligned to 16; n numbers exist, the others are 0
template <typename T, int Q>
struct RowPart {
  static constexpr int P = 16 / (int)sizeof(T), N = Q * P;
  uint4 q[Q];
  __device__ __forceinline__ void load(const T* p, int n) {
#pragma unroll
    for (int k = 0; k < Q; ++k) {
      q[k] = make_uint4(0, 0, 0, 0);
      const int left = n - k * P;
      if (left >= P) {
        q[k] = reinterpret_cast<const uint4*>(p)[k];
      } else if (left > 0) {
        uint32_t w[4] = {};
#pragma unroll
        for (int i = 0; i < P; ++i)
          if (i < left) {
            if constexpr (sizeof(T) == 2) w[i / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[k * P + i] << (16 * (i & 1));
            else w[i] = reinterpret_cast<const uint32_t*>(p)[k * P + i];
          }
        q[k] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
  }
  __device__ __forceinline__ void unpack(float* v) const {
#pragma unroll
    for (int k = 0; k < Q; ++k) {
      const uint32_t w[4] = {q[k].x, q[k].y, q[k].z, q[k].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 2) v[k * P + 2 * i] = __uint_as_float(w[i] << 16), v[k * P + 2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        else v[k * P + i] = __uint_as_float(w[i]);
      }
    }
  }
};
// A lane's part: 32 bytes; 16 of bf16 where there is a z, too, so that three CTAs share an SM and two tokens of a warp are on their way (8192 x 16384 with gelu_tanh 173 us; 32 bytes
// and two CTAs 192, 16 bytes and four CTAs with one token on its way 182).
template <typename T, bool HAS_Z>
using RowOf = RowPart<T, sizeof(T) == 2 && HAS_Z ? 1 : 2>;
constexpr int kAhead = 2;

template <typename T, bool CL, bool HAS_Z>
__global__ void __launch_bounds__(256, 3) act_backward_kernel(const ActBwdArgs p) {
  grid_started();
  grid_ready();
  using Row = RowOf<T, HAS_Z>;
  constexpr int N = Row::N;
  __shared__ float part[8 * 32 * N];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, first = blockIdx.x * (32 * N), at = first + lane * N, n = p.d - at;
  const int64_t end = min(p.t, (blockIdx.y + 1) * p.per);
  const T* dy = static_cast<const T*>(p.DY) + at;
  const T* z = static_cast<const T*>(p.Z) + at;
  float sum[N] = {};
  Row ny[kAhead], nz[HAS_Z ? kAhead : 1];  // what is on its way
  int64_t t = blockIdx.y * p.per + warp;
#pragma unroll
  for (int u = 0; u < kAhead; ++u) ny[u].load(dy + (t + 8 * u) * p.lddy, t + 8 * u < end ? n : 0);
  if constexpr (HAS_Z) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) nz[u].load(z + (t + 8 * u) * p.ldz, t + 8 * u < end ? n : 0);
  }
  for (; t < end; t += 8) {
    float v[N];
    const int64_t next = t + 8 * kAhead;
    ny[0].unpack(v);
#pragma unroll
    for (int u = 1; u < kAhead; ++u) ny[u - 1] = ny[u];
    if constexpr (HAS_Z) {
      float w[N];
      nz[0].unpack(w);
#pragma unroll
      for (int u = 1; u < kAhead; ++u) nz[u - 1] = nz[u];
      nz[kAhead - 1].load(z + next * p.ldz, next < end ? n : 0);
      ny[kAhead - 1].load(dy + next * p.lddy, next < end ? n : 0);
      act_slopes<N>(p.act, v, w);
    } else {
      ny[kAhead - 1].load(dy + next * p.lddy, next < end ? n : 0);
    }
#pragma unroll
    for (int j = 0; j < N; j += 2) {
      const Two s = add2({sum[j], sum[j + 1]}, {v[j], v[j + 1]});
      sum[j] = s.a, sum[j + 1] = s.b;
    }
    if (p.DZ) {
      T* to = static_cast<T*>(p.DZ) + t * p.lddz + at;
#pragma unroll
      for (int j = 0; j < N; j += 8) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = v[j + e];
        store8(to + j, n - j, true, x);
      }
    }
    if (p.Q) {
      float m = fabsf(v[0]);
#pragma unroll
      for (int j = 1; j < N; ++j) m = larger_nan(m, fabsf(v[j]));
#pragma unroll
      for (int o = 64 / N; o > 0; o >>= 1) m = larger_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
      const uint32_t byte = f8_scale_byte(__float_as_uint(m));
      if (n > 0) {
        const float inv = byte == kScaleNan ? 0.0f : f8_inv_scale(byte);
        uint32_t q[N / 4];
#pragma unroll
        for (int j = 0; j < N; j += 4) {
          const Two a = mul2({v[j], v[j + 1]}, both(inv)), b = mul2({v[j + 2], v[j + 3]}, both(inv));
          q[j / 4] = byte == kScaleNan ? 0x7f7f7f7fu : f8_pack4(a.a, a.b, b.a, b.b);
        }
        uint8_t* to = static_cast<uint8_t*>(p.Q) + t * p.ldq + at;
#pragma unroll
        for (int j = 0; j < N; j += 8) store8_f8(to + j, n - j, true, make_uint2(q[j / 4], q[j / 4 + 1]));
        if ((lane & (kF8Block / N - 1)) == 0) static_cast<uint8_t*>(p.S)[t * p.lds + at / kF8Block] = (uint8_t)byte;
      }
    }
  }
  if (!p.sums) return;
#pragma unroll
  for (int j = 0; j < N; j += 4) *reinterpret_cast<float4*>(part + warp * 32 * N + lane * N + j) = make_float4(sum[j], sum[j + 1], sum[j + 2], sum[j + 3]);
  act_sum_up<CL>(p, part, 32 * N, first);
}

// Columns that start anywhere: lanes read neighbouring numbers one by one, 256 features of a token a warp.
template <typename T, bool CL>
__global__ void __launch_bounds__(256, 3) act_backward_anywhere_kernel(const ActBwdArgs p) {
  grid_started();
  grid_ready();
  using Piece = Warp256<T, false>;
  __shared__ float part[8 * 256];
  const int warp = threadIdx.x >> 5, first = blockIdx.x * 256;
  const int64_t end = min(p.t, (blockIdx.y + 1) * p.per);
  float sum[8] = {};
  for (int64_t t0 = blockIdx.y * p.per + warp; t0 < end; t0 += 8 * kTokens) {
    Raw8<T> dy[kTokens], z[kTokens];
#pragma unroll
    for (int u = 0; u < kTokens; ++u) {
      const int64_t t = t0 + 8 * u;
      const int n = t < end ? p.d : 0;
      Piece::load(static_cast<const T*>(p.DY) + (t < end ? t : t0) * p.lddy, first, n, dy[u]);
      if (p.Z) Piece::load(static_cast<const T*>(p.Z) + (t < end ? t : t0) * p.ldz, first, n, z[u]);
    }
#pragma unroll
    for (int u = 0; u < kTokens; ++u) {
      const int64_t t = t0 + 8 * u;
      if (t >= end) break;
      float v[8], w[8];
      unpack8(dy[u], v);
      if (p.Z) {
        unpack8(z[u], w);
        act_slopes<8>(p.act, v, w);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[j] += v[j];  // beyond the token's end dy is 0 and so is z, whose derivative is finite
      if (p.DZ) Piece::store(static_cast<T*>(p.DZ) + t * p.lddz, first, p.d, v);
      if (p.Q) Piece::quantise(v, static_cast<uint8_t*>(p.Q) + t * p.ldq, static_cast<uint8_t*>(p.S) + t * p.lds, first, p.d);
    }
  }
  if (!p.sums) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) part[warp * 256 + Piece::index(0, j)] = sum[j];
  act_sum_up<CL>(p, part, 256, first);
}

__global__ void __launch_bounds__(256) act_sum_kernel(const float* sums, int parts, int d, float* db) {
  grid_started();
  grid_ready();
  __shared__ float part[8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.x * 32 + lane;
  float s = 0.0f;
  if (i < d)
    for (int k = warp; k < parts; k += 8) s += sums[k * (int64_t)d + i];
  part[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && i < d) {
#pragma unroll
    for (int k = 1; k < 8; ++k) s += part[k][lane];
    db[i] = s;
  }
}

// Tokens of a CTA and CTAs to the same features, counted with 512 features to a CTA for every kind of columns: as many CTAs as the SMs hold at once, three each.  Few tokens are
// shared by a cluster of up to eight, which adds up by itself; where there would be a few more than that, by eight.
struct ActSplit {
  int64_t per;
  unsigned parts;
};
ActSplit act_split(int64_t d, int64_t t) {
  const int64_t room = (int64_t)sm_count_cached() * 3 / blocks_of(d, 512), wanted = room < 1 ? 1 : room;
  int64_t per = blocks_of(blocks_of(t, wanted), 8) * 8;
  if (per < 32) per = 32;  // four tokens a warp
  if (blocks_of(t, per) < 2 * kMostCluster && blocks_of(t, per) * blocks_of(d, 512) < sm_count_cached() * 2) per = blocks_of(blocks_of(t, kMostCluster), 8) * 8;
  int64_t parts = blocks_of(t, per);
  if (parts > 65535) per = blocks_of(t, 65535), parts = blocks_of(t, per);
  return {per, (unsigned)parts};
}

template <typename T>
int act_backward_launch(const ActBwdArgs& a, bool vec, unsigned parts, bool cluster, cudaStream_t st) {
  const dim3 grid((unsigned)blocks_of(a.d, !vec ? 256 : 32 * (a.Z ? RowOf<T, true>::N : RowOf<T, false>::N)), parts);
  if (!vec) {
    if (cluster) return launch_overlapped_as(act_backward_anywhere_kernel<T, true>, grid, 256, 0, dim3(1, parts), st, a);
    return launch_overlapped(act_backward_anywhere_kernel<T, false>, grid, 256, st, a);
  }
  if (cluster) return launch_overlapped_as(a.Z ? act_backward_kernel<T, true, true> : act_backward_kernel<T, true, false>, grid, 256, 0, dim3(1, parts), st, a);
  return launch_overlapped(a.Z ? act_backward_kernel<T, false, true> : act_backward_kernel<T, false, false>, grid, 256, st, a);
}

}  // namespace
}  // namespace b2

extern "C" size_t b2_act_backward_workspace_bytes(int64_t d, int64_t t) {
  using namespace b2;
  if (d <= 0 || t <= 0 || d > kMostFeatures) return 0;
  const ActSplit s = act_split(d, t);
  return s.parts > kMostCluster ? round_up((size_t)s.parts * (size_t)d * 4, 256) : 0;
}

extern "C" int b2_act_backward(int64_t d, int64_t t, int type, int act, const void* DY, int64_t lddy, const void* Z, int64_t ldz, void* DZ,
                               int64_t lddz, void* Q, int64_t ldq, void* S, int64_t lds, float* db, void* workspace, size_t workspace_bytes,
                               void* cuda_stream) {
  using namespace b2;
  if (d < 0) return -1;
  if (t < 0) return -2;
  if (type != B2_TYPE_F32 && type != B2_TYPE_BF16) return -3;
  if (!act_known(act)) return -4;
  const bool work = d > 0 && t > 0;
  const int64_t least = d > 1 ? d : 1;
  if (act == B2_ACT_NONE) Z = nullptr;
  if (work && !DY) return -5;
  if (lddy < least) return -6;
  if (work && act != B2_ACT_NONE && !Z) return -7;
  if (Z && ldz < least) return -8;
  if (DZ && lddz < least) return -10;
  if (Q && ldq < least) return -12;
  if (work && Q && !S) return -13;
  if (Q && lds < (d > 0 ? blocks_of(d, kF8Block) : 1)) return -14;
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  if (d > 0 && db && t == 0) return cudaMemsetAsync(db, 0, (size_t)d * 4, st) == cudaSuccess ? B2_OK : B2_ERR_LAUNCH;
  if (!work || (!DZ && !Q && !db)) return B2_OK;
  if (d > kMostFeatures) return B2_ERR_VARIANT;
  const ActSplit s = act_split(d, t);
  const bool partial = db && s.parts > kMostCluster, cluster = db && s.parts > 1 && !partial;
  if (partial && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0 || workspace_bytes < b2_act_backward_workspace_bytes(d, t)))
    return B2_ERR_WORKSPACE;
  const int es = type == B2_TYPE_BF16 ? 2 : 4;
  const ActBwdArgs a{(int)d, act, t, s.per, DY, Z, DZ, Q, S, lddy, ldz, lddz, ldq, lds, partial ? static_cast<float*>(workspace) : db};
  const bool vec = columns_aligned(DY, lddy, es, 16) && (!Z || columns_aligned(Z, ldz, es, 16)) && (!DZ || columns_aligned(DZ, lddz, es, 16)) &&
                   (!Q || columns_aligned(Q, ldq, 1, 8));
  const int rc = type == B2_TYPE_BF16 ? act_backward_launch<__nv_bfloat16>(a, vec, s.parts, cluster, st) : act_backward_launch<float>(a, vec, s.parts, cluster, st);
  if (rc || !partial) return rc;
  return launch_overlapped(act_sum_kernel, (unsigned)blocks_of(d, 32), 256, st, static_cast<const float*>(workspace), (int)s.parts, (int)d, db);
}
