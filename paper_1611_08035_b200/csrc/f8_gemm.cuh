// Arguments of the block-scaled e4m3 product, shared by its kernels.
#pragma once
#include <cuda.h>

#include "b2gemm.h"
#include "entry.h"
#include "f8.cuh"
#include "f8_out.cuh"
#include "tcgen05.cuh"

namespace b2 {

constexpr int kRows = 128;                       // MMA rows of a CTA's tile
constexpr uint32_t kRowStage = kRows * kF8Block;  // bytes of the row operand in a stage
constexpr int kMaxSplit = 8;

struct F8Scale {  // value for index i and block b: p[(i >> shift) * si + b * sb]
  const void* p;
  int64_t si, sb;
  int shift, f32;
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

// Matrix of bytes, `inner` contiguous; boxes of 128 bytes by box_outer, 128-byte swizzle.
inline bool f8_map(CUtensorMap* map, const void* base, int64_t inner, int64_t outer, int64_t ld, int box_outer) {
  EncodeFn enc = tensor_map_encode_fn();
  if (!enc) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)outer};
  const cuuint64_t strides[1] = {(cuuint64_t)ld};
  const cuuint32_t box[2] = {128, (cuuint32_t)box_outer};
  const cuuint32_t estr[2] = {1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}


// f8_mx.cu: products whose scales are both e8m0, 256 x 256 tiles; TC = float or __nv_bfloat16
template <typename TC>
int f8_mx_launch(F8Args a, const F8Operand& r, const F8Operand& c, int64_t k, cudaStream_t st);

}  // namespace b2
