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

// The same for a warp whose lanes own 32 consecutive rows (row0 + lane) and N consecutive columns each, columns
// contiguous and aligned in C.  64 bytes of every row pass through shared memory at a time and leave as whole 64-byte pieces
// of eight rows an instruction: a lane that stores its own row directly touches 32 lines with every instruction (a 256 x 256
// bf16 tile: 8000 clocks of storing, as long as the multiply-adds of 2000 summed elements).
constexpr int kEmitPitch = 80;  // bytes between staged rows: 16-byte pieces of eight rows in different banks
constexpr int kEmitBytes = 32 * kEmitPitch;
template <typename TC, int N>
__device__ __forceinline__ void f8_emit_staged(const F8Out& p, int64_t row0, int64_t col0, const float* acc, unsigned char* stage) {
  const int lane = threadIdx.x & 31, piece = lane & 3;
  TC* C = static_cast<TC*>(p.C);
  unsigned char* own = stage + lane * kEmitPitch;
  const unsigned char* swap = stage + (lane >> 2) * kEmitPitch + piece * 16;
  if (sizeof(TC) == 2 && p.beta == 0.0f) {
#pragma unroll
    for (int j = 0; j < N; j += 32) {
      __syncwarp();
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float* a = acc + j + 8 * i;
        *reinterpret_cast<uint4*>(own + 16 * i) = make_uint4(pack_bf16(p.alpha * a[0], p.alpha * a[1]), pack_bf16(p.alpha * a[2], p.alpha * a[3]),
                                                             pack_bf16(p.alpha * a[4], p.alpha * a[5]), pack_bf16(p.alpha * a[6], p.alpha * a[7]));
      }
      __syncwarp();
      const int64_t col = col0 + j + piece * 8, nv = p.cols - col;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t row = row0 + 8 * i + (lane >> 2);
        const uint4 q = *reinterpret_cast<const uint4*>(swap + 8 * i * kEmitPitch);
        if (row < p.rows) {
          if (nv >= 8) {
            *reinterpret_cast<uint4*>(C + row * p.ldc + col) = q;
          } else {
            const uint32_t w[4] = {q.x, q.y, q.z, q.w};
            uint16_t* c = reinterpret_cast<uint16_t*>(C + row * p.ldc + col);
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (e < nv) c[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
          }
        }
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; j += 16) {
      __syncwarp();
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4*>(own + 16 * i) = make_float4(p.alpha * acc[j + 4 * i], p.alpha * acc[j + 4 * i + 1], p.alpha * acc[j + 4 * i + 2], p.alpha * acc[j + 4 * i + 3]);
      __syncwarp();
      const int64_t col = col0 + j + piece * 4, nv = p.cols - col;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t row = row0 + 8 * i + (lane >> 2);
        const float4 q = *reinterpret_cast<const float4*>(swap + 8 * i * kEmitPitch);
        float v[4] = {q.x, q.y, q.z, q.w};
        if (row < p.rows) {
          TC* c = C + row * p.ldc + col;
          if (p.beta != 0.0f) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (e < nv) v[e] += p.beta * f8_load1(c + e);
          }
          if (sizeof(TC) == 4 && nv >= 4) {
            *reinterpret_cast<float4*>(c) = make_float4(v[0], v[1], v[2], v[3]);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (e < nv) f8_store1(c + e, v[e]);
          }
        }
      }
    }
  }
}

// Joining the shares of a k split: the CTAs of a cluster (rank = share) have each put their part of the 128 x TBN tile
// into their shared memory as floats [column][row]; each adds all parts, in the order of the ranks, for its columns.  All
// threads of all CTAs of the cluster call this; warps with writer >= 0 (0 .. EW-1, covering the tensor-memory lanes 32 *
// quad .. + 31) add and write; `row` is the row of C that this lane's accumulators belong to.
template <typename TC, bool COLS_CONTIG, int TBN, int EW>
__device__ __forceinline__ void f8_split_join(const F8Out& p, const void* tile, int splits, int share, int writer, int quad,
                                              int64_t row, int64_t col0) {
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
      f8_emit<TC, COLS_CONTIG, G>(p, row, col0 + c, v);
    }
  }
  __syncwarp();
  cluster_sync_all();  // no CTA leaves while another one reads its share
}

// C := beta * C, and copies of operands into 16-byte aligned columns (ldd a multiple of 16 bytes); defined in f8_gemm.cu.
int f8_scale_c(int64_t m, int64_t n, float beta, void* C, int64_t ldc, int type_c, cudaStream_t st);
int f8_repitch(const void* src, int64_t ld_bytes, int64_t row_bytes, int64_t cols, void* dst, int64_t ldd_bytes, cudaStream_t st);

}  // namespace b2
