// The backward pass of an activation and a bias:
//
//   dz = dy act'(z),   db_i = sum over tokens of dz_i,   (q, s) = dz quantised in blocks of 128 features of a token
//
// Bound by memory: dy and z are read once, dz and q written once.  A warp holds 256 consecutive features (two blocks of 128) of kTokens tokens at a time; all
// their loads are issued before the first is used.  The eight warps of a CTA take the same features of different tokens, so that a feature's sum
// stays in one lane's register over all of a warp's tokens, and what is left to add are eight numbers a CTA and one a CTA of the same features, in a fixed order.
#include "act.cuh"
#include "b2gemm.h"
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
constexpr int kTokens = 2;  // of a warp at a time

template <typename T, bool VEC>
__global__ void __launch_bounds__(256, 3) act_backward_kernel(const ActBwdArgs p) {
  grid_started();
  grid_ready();
  using Piece = Warp256<T, VEC>;
  __shared__ float part[8][256];
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
  for (int j = 0; j < 8; ++j) part[warp][Piece::index(0, j)] = sum[j];
  __syncthreads();
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) s += part[i][threadIdx.x];
  if (first + (int)threadIdx.x < p.d) p.sums[blockIdx.y * (int64_t)p.d + first + threadIdx.x] = s;
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

// Tokens of a CTA and CTAs to the same features: as many as it takes to give every SM several, but not fewer tokens than its warps have under way at once,
// twice over; one CTA, whose sums are the result, as long as that is 64 tokens.
struct ActSplit {
  int64_t per;
  unsigned parts;
};
ActSplit act_split(int64_t d, int64_t t) {
  const int64_t wanted = blocks_of((int64_t)sm_count_cached() * 9, blocks_of(d, 256));
  int64_t per = blocks_of(blocks_of(t, wanted), 8 * kTokens) * 8 * kTokens;
  if (per < 64) per = 64;
  int64_t parts = blocks_of(t, per);
  if (parts > 65535) per = blocks_of(t, 65535), parts = blocks_of(t, per);
  return {per, (unsigned)parts};
}

template <typename T>
int act_backward_launch(const ActBwdArgs& a, bool vec, dim3 grid, cudaStream_t st) {
  return vec ? launch_overlapped(act_backward_kernel<T, true>, grid, 256, st, a) : launch_overlapped(act_backward_kernel<T, false>, grid, 256, st, a);
}

}  // namespace
}  // namespace b2

extern "C" size_t b2_act_backward_workspace_bytes(int64_t d, int64_t t) {
  using namespace b2;
  if (d <= 0 || t <= 0 || d > kMostFeatures) return 0;
  const ActSplit s = act_split(d, t);
  return s.parts > 1 ? round_up((size_t)s.parts * (size_t)d * 4, 256) : 0;
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
  const bool partial = db && s.parts > 1;
  if (partial && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0 || workspace_bytes < b2_act_backward_workspace_bytes(d, t)))
    return B2_ERR_WORKSPACE;
  const int es = type == B2_TYPE_BF16 ? 2 : 4;
  const ActBwdArgs a{(int)d, act, t, s.per, DY, Z, DZ, Q, S, lddy, ldz, lddz, ldq, lds, partial ? static_cast<float*>(workspace) : db};
  const bool vec = columns_aligned(DY, lddy, es, 16) && (!Z || columns_aligned(Z, ldz, es, 16)) && (!DZ || columns_aligned(DZ, lddz, es, 16)) &&
                   (!Q || columns_aligned(Q, ldq, 1, 8));
  const dim3 grid((unsigned)blocks_of(d, 256), s.parts);
  const int rc = type == B2_TYPE_BF16 ? act_backward_launch<__nv_bfloat16>(a, vec, grid, st) : act_backward_launch<float>(a, vec, grid, st);
  if (rc || !partial) return rc;
  return launch_overlapped(act_sum_kernel, (unsigned)blocks_of(d, 32), 256, st, static_cast<const float*>(workspace), (int)s.parts, (int)d, db);
}
