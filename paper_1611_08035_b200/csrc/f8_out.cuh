// The end of the 8-bit products: C := alpha * acc + beta * C from accumulators in registers, and the sum over the CTAs
// of a cluster that share a tile's k range.
#pragma once
#include "common.cuh"
#include "f8.cuh"

namespace b2 {

struct F8Out {
  int64_t rows, cols;  // extents of the MMA's row and column index
  float alpha, beta;
  void* C;
  int64_t ldc;
  int vec;  // columns of C are 16-byte aligned
};

// alpha * v + beta * old for 8 (or fewer) consecutive elements
template <typename TC>
__device__ __forceinline__ void f8_emit8(TC* c, int64_t nv, bool vec, float alpha, float beta, float (&v)[8]) {
  if (beta != 0.0f) {
    float old[8];
    load8(c, nv, vec, old);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = alpha * v[j] + beta * old[j];
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= alpha;
  }
  store8(c, nv, vec, v);
}
__device__ __forceinline__ float f8_load1(const float* p) { return *p; }
__device__ __forceinline__ float f8_load1(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void f8_store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void f8_store1(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// N (a multiple of 8, or any count with rows contiguous) accumulators of one row.  COLS_CONTIG: C[row * ldc + col].
template <typename TC, bool COLS_CONTIG, int N>
__device__ __forceinline__ void f8_emit(const F8Out& p, int64_t row, int64_t col, const float* acc) {
  if (row >= p.rows) return;
  TC* C = static_cast<TC*>(p.C);
  if constexpr (COLS_CONTIG) {
#pragma unroll
    for (int j = 0; j < N; j += 8) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = acc[j + i];
      f8_emit8(C + row * p.ldc + col + j, p.cols - col - j, p.vec != 0, p.alpha, p.beta, v);
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (col + j < p.cols) {
        TC* c = C + (col + j) * p.ldc + row;
        float v = p.alpha * acc[j];
        if (p.beta != 0.0f) v += p.beta * f8_load1(c);
        f8_store1(c, v);
      }
    }
  }
}

// Joining the shares of a k split: the CTAs of a cluster (rank = share) have each put their part of the 128 x TBN tile
// into their shared memory as floats [column][row]; each adds all parts, in the order of the ranks, for its columns.  All
// threads of all CTAs of the cluster call this; warps with writer >= 0 (0 .. EW-1, covering the tensor-memory lanes 32 *
// quad .. + 31) add and write.
template <typename TC, bool COLS_CONTIG, int TBN, int EW>
__device__ __forceinline__ void f8_split_join(const F8Out& p, const void* tile, int splits, int share, int writer, int quad,
                                              int64_t row0, int64_t col0) {
  cluster_sync_all();
  if (writer >= 0) {
    const int lane = threadIdx.x & 31;
    const int per = TBN / splits / (EW / 4), c_first = share * (TBN / splits) + (writer >> 2) * per;
    constexpr int G = COLS_CONTIG ? 8 : 2;
    for (int c = c_first; c < c_first + per; c += G) {
      float v[G];
#pragma unroll
      for (int g = 0; g < G; ++g) v[g] = 0.0f;
      for (int q = 0; q < splits; ++q) {
        const uint32_t base = cluster_map_shared(smem_u32(tile), (uint32_t)q);
#pragma unroll
        for (int g = 0; g < G; ++g) {
          float x;
          asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(base + (uint32_t)(((c + g) * 128 + quad * 32 + lane) * 4)) : "memory");
          v[g] += x;
        }
      }
      f8_emit<TC, COLS_CONTIG, G>(p, row0 + quad * 32 + lane, col0 + c, v);
    }
  }
  __syncwarp();
  cluster_sync_all();  // no CTA leaves while another one reads its share
}

// C := beta * C, and copies of operands into 16-byte aligned columns (ldd a multiple of 16 bytes); defined in f8_gemm.cu.
int f8_scale_c(int64_t m, int64_t n, float beta, void* C, int64_t ldc, int type_c, cudaStream_t st);
int f8_repitch(const void* src, int64_t ld_bytes, int64_t row_bytes, int64_t cols, void* dst, int64_t ldd_bytes, cudaStream_t st);

}  // namespace b2
