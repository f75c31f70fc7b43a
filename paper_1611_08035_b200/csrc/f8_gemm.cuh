// Arguments of the block-scaled e4m3 product, shared by its kernels.
#pragma once
#include <cuda.h>

#include <atomic>

#include "b2gemm.h"
#include "entry.h"
#include "f8.cuh"
#include "f8_out.cuh"
#include "tcgen05.cuh"

namespace b2 {

constexpr int kRows = 128;                       // MMA rows of a CTA's tile
constexpr uint32_t kRowStage = kRows * kF8Block;  // bytes of the row operand in a stage

struct F8Scale {  // value for index i and block b: p[(i >> shift) * si + b * sb]
  const void* p;
  int64_t si, sb;
  int shift, f32;
  int words;  // bytes, four consecutive blocks at a time in aligned words
};
struct F8Args {
  F8Out out;
  int kb;              // blocks of 128 along the summed index
  int splits;          // CTAs of a cluster that share a tile's blocks
  int r_mn, c_mn;      // the operand's own index is contiguous (else the summed one)
  int tiles_r, tiles_c, group;
  F8Scale sr, sc;
  int* status;
};

__device__ __forceinline__ float f8_scale_at(const F8Scale& s, int64_t i, int b) {
  const int64_t at = (i >> s.shift) * s.si + (int64_t)b * s.sb;
  return s.f32 ? static_cast<const float*>(s.p)[at] : e8m0_value(static_cast<const uint8_t*>(s.p)[at]);
}

struct F8Operand {
  const void* p;
  int64_t n, ld;  // extent of its own index, leading dimension
  bool mn;        // its own index is contiguous
  F8Scale s;
};

// Blocks whose products are summed in tensor memory before the sum moves to fp32 registers.  The tensor core's additions truncate, so
// that a sum which grows for long comes out too small: fp32 results over k = 262144, eight shares of 32768, were 1.8e-5 off (all terms of one sign,
// mean), 32000 x 8 over 65536 without a split 5.9e-5; moved every 2048 the mean is 1e-6 and does not grow.  bf16, whose rounding is 2e-3, sees
// sums over 65536 (6e-5), and without a limit 1.4e-3 at k = 4194304.
template <typename TC>
__host__ __device__ constexpr int chunk_blocks() { return sizeof(TC) == 4 ? 16 : 512; }

// Matrix of bytes, `inner` contiguous; boxes of box_inner (128 or 64) bytes by box_outer, swizzled over their width.
inline bool f8_map(CUtensorMap* map, const void* base, int64_t inner, int64_t outer, int64_t ld, int box_outer, int box_inner = 128) {
  EncodeFn enc = tensor_map_encode_fn();
  if (!enc) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)outer};
  const cuuint64_t strides[1] = {(cuuint64_t)ld};
  const cuuint32_t box[2] = {(cuuint32_t)box_inner, (cuuint32_t)box_outer};
  const cuuint32_t estr[2] = {1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, box_inner == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Instruction descriptor: fp32 accumulator, e4m3 operands (format 0), which of them have their own index contiguous, N, M.
__device__ __forceinline__ uint32_t umma_idesc_f8(int m, int n, int a_mn, int b_mn) {
  return (1u << 4) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

// Instruction descriptor: byte of the scale words (both operands), e4m3, which operands have their own index contiguous,
// N, e8m0 scales, M.
__device__ __forceinline__ uint32_t umma_idesc_mx(int m, int n, int a_mn, int b_mn, int byte) {
  return ((uint32_t)byte << 4) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) | (1u << 23) |
         ((uint32_t)(m >> 7) << 27) | ((uint32_t)byte << 29);
}

// Scale bytes of the indices i, i + 32, .. (clamped to the last one) for blocks b .. b+3, b a multiple of four, the first in the lowest
// byte; blocks beyond the last are never multiplied with.  All loads come before the first use: joined one word after the other, the bytes of
// 38 blocks kept a 512 x 512 product 10.6 us where 32 blocks, read in words, took 7.8.
template <int N>
__device__ __forceinline__ void scale_words(const F8Scale& s, int64_t i, int64_t extent, int b, int kb, uint32_t* w) {
  const uint8_t* p[N];
#pragma unroll
  for (int n = 0; n < N; ++n)
    p[n] = static_cast<const uint8_t*>(s.p) + ((i + 32 * n < extent ? i + 32 * n : extent - 1) >> s.shift) * s.si + (int64_t)b * s.sb;
  if (s.words && b + 4 <= kb) {
#pragma unroll
    for (int n = 0; n < N; ++n) w[n] = *reinterpret_cast<const uint32_t*>(p[n]);
  } else {
    uint32_t v[N][4];
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j) v[n][j] = b + j < kb ? p[n][j * s.sb] : 0u;
#pragma unroll
    for (int n = 0; n < N; ++n) w[n] = v[n][0] | v[n][1] << 8 | v[n][2] << 16 | v[n][3] << 24;
  }
}

// Launch of a persistent kernel on pairs of CTAs with 256 x 256 tiles.
template <typename Kernel>
int f8_pair_launch(Kernel kfn, std::atomic<bool>* configured, int threads, size_t smem, F8Args a, const F8Operand& r, const F8Operand& c,
                   int64_t k, cudaStream_t st) {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return B2_ERR_LAUNCH;
  if (!configured[dev].load(std::memory_order_acquire)) {
    if (cudaFuncSetAttribute(kfn, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return B2_ERR_LAUNCH;
    configured[dev].store(true, std::memory_order_release);
  }
  CUtensorMap mr, mc;
  if (!f8_map(&mr, r.p, r.mn ? r.n : k, r.mn ? k : r.n, r.ld, 128) || !f8_map(&mc, c.p, c.mn ? c.n : k, c.mn ? k : c.n, c.ld, 128))
    return B2_ERR_LAUNCH;
  const int64_t tr = blocks_of(r.n, 256), tc = blocks_of(c.n, 256);
  if (tr * tc > 0x3fffffffLL) return B2_ERR_VARIANT;
  a.out.rows = r.n, a.out.cols = c.n, a.r_mn = r.mn, a.c_mn = c.mn, a.sr = r.s, a.sc = c.s;
  a.tiles_r = (int)tr, a.tiles_c = (int)tc, a.splits = 1, a.group = 8;
  const int tiles = a.tiles_r * a.tiles_c, pairs = sm_count_cached() / 2;
  return launch_overlapped_as(kfn, dim3(2u * (unsigned)(tiles < pairs ? tiles : pairs)), (unsigned)threads, smem, dim3(2), st, a, mr, mc);
}

// f8_mx.cu: products whose scales are both e8m0, 256 x 256 tiles; TC = float or __nv_bfloat16
template <typename TC>
int f8_mx_launch(F8Args a, const F8Operand& r, const F8Operand& c, int64_t k, cudaStream_t st);
// f8_fs.cu: the same with scales of either type
template <typename TC>
int f8_fs_launch(F8Args a, const F8Operand& r, const F8Operand& c, int64_t k, cudaStream_t st);

}  // namespace b2
