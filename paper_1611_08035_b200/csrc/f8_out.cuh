// The end of the 8-bit products: C := alpha * acc + beta * C from accumulators in registers, and the sum over the CTAs
// of a cluster that share a tile's k range.
#pragma once
#include "common.cuh"
#include "f8.cuh"
#include "tcgen05.cuh"

namespace b2 {

struct F8Out {
  int64_t rows, cols;  // extents of the MMA's row and column index
  float alpha, beta;
  void* C;
  int64_t ldc;
  int vec;  // columns of C are 16-byte aligned
};

__device__ __forceinline__ float f8_load1(const float* p) { return *p; }
__device__ __forceinline__ float f8_load1(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void f8_store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void f8_store1(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void f8_load4(const float* p, float v[4]) {
  const float4 q = *reinterpret_cast<const float4*>(p);
  v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
}
__device__ __forceinline__ void f8_load4(const __nv_bfloat16* p, float v[4]) {
  const uint2 q = *reinterpret_cast<const uint2*>(p);
  v[0] = __uint_as_float(q.x << 16), v[1] = __uint_as_float(q.x & 0xffff0000u);
  v[2] = __uint_as_float(q.y << 16), v[3] = __uint_as_float(q.y & 0xffff0000u);
}
__device__ __forceinline__ void f8_store4(float* p, const float v[4]) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }
__device__ __forceinline__ void f8_store4(__nv_bfloat16* p, const float v[4]) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
}

// Old values of `lines` runs of C on their way to L2 while the tile is computed: run i starts at element (outer + i) of the index that is not
// contiguous in C and `first` of the one that is, and has `count` elements.  A warp's lanes share the runs.
// 8192 x 8192 with beta: product over 256, fp32 scales, bf16 121 -> 108 us, fp32 161 -> 123, e8m0 bf16 104 -> 94; weight gradient over 4096 tokens
// bf16 606 -> 484.  Not used by the e8m0 product in fp32, whose registers it takes from results without beta (78 -> 80.5 us), nor by
// the weight gradient in fp32 (210 -> 237 over 256 tokens: its old values are then asked for too early).
template <typename TC>
__device__ __forceinline__ void f8_prefetch(const F8Out& p, bool cols_contiguous, int64_t outer, int lines, int64_t first, int count) {
  if (p.beta == 0.0f) return;
  const int64_t outers = cols_contiguous ? p.rows : p.cols, inners = cols_contiguous ? p.cols : p.rows;
  for (int i = threadIdx.x & 31; i < lines; i += 32)
    for (int e = 0; e < count; e += 128 / (int)sizeof(TC))
      if (outer + i < outers && first + e < inners)
        asm volatile("prefetch.global.L2 [%0];" ::"l"(static_cast<const TC*>(p.C) + (outer + i) * p.ldc + first + e));
}

// N accumulators of one row of a tile whose rows are contiguous in C (C[col * ldc + row]): neighbouring lanes, neighbouring rows.
// Straight code with one test of beta: with one at every column a tile's 64 columns a warp took 4 us (a gradient of 4096 x 4096 over
// 64 tokens 36 us, now 21).
template <typename TC, int N>
__device__ __forceinline__ void f8_emit_rows(const F8Out& p, int64_t row, int64_t col, float* acc) {
  float beta = p.beta;
  int64_t ldc = p.ldc;
  asm volatile("" : "+f"(beta), "+l"(ldc));  // what follows from these is not kept in registers over the loop that fills acc
  const int nv = row < p.rows ? (int)min((int64_t)N, p.cols - col) : 0;
  TC* C = static_cast<TC*>(p.C) + row + col * ldc;
  if (beta != 0.0f) {
#pragma unroll
    for (int j0 = 0; j0 < N; j0 += 8) {
      float old[8];
      const TC* c = C + j0 * ldc;
#pragma unroll
      for (int j = 0; j < 8; ++j, c += ldc) old[j] = j0 + j < nv ? f8_load1(c) : 0.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j0 + j] = p.alpha * acc[j0 + j] + beta * old[j];
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) acc[j] *= p.alpha;
  }
#pragma unroll
  for (int j = 0; j < N; ++j, C += ldc)
    if (j < nv) f8_store1(C, acc[j]);
}

// N consecutive accumulators each of 32 consecutive rows (row0 + lane), columns contiguous in C.  64 bytes of every row pass through shared memory at a time and leave as whole 64-byte pieces
// of eight rows an instruction: a lane that stores its own row directly touches 32 lines with every instruction (a 256 x 256
// bf16 tile: 8000 clocks of storing, as long as the multiply-adds of 2000 summed elements).
constexpr int kEmitPitch = 80;  // bytes between staged rows: 16-byte pieces of eight rows in different banks
constexpr int kEmitBytes = 32 * kEmitPitch;
template <typename TC, int N>
__device__ __forceinline__ void f8_emit_staged(const F8Out& p, int64_t row0, int64_t col0, const float* acc, unsigned char* stage) {
  float beta = p.beta;
  int64_t ldc = p.ldc;
  asm volatile("" : "+f"(beta), "+l"(ldc));  // what follows from these is not kept in registers over the loop that fills acc
  const int lane = threadIdx.x & 31, piece = lane & 3;
  TC* C = static_cast<TC*>(p.C);
  unsigned char* own = stage + lane * kEmitPitch;
  const unsigned char* swap = stage + (lane >> 2) * kEmitPitch + piece * 16;
  if (sizeof(TC) == 2 && beta == 0.0f && p.vec) {
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
            *reinterpret_cast<uint4*>(C + row * ldc + col) = q;
          } else {
            const uint32_t w[4] = {q.x, q.y, q.z, q.w};
            uint16_t* c = reinterpret_cast<uint16_t*>(C + row * ldc + col);
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (e < nv) c[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
          }
        }
      }
    }
    return;
  }
  auto put = [&](int j) {
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<float4*>(own + 16 * i) = make_float4(p.alpha * acc[j + 4 * i], p.alpha * acc[j + 4 * i + 1], p.alpha * acc[j + 4 * i + 2], p.alpha * acc[j + 4 * i + 3]);
    __syncwarp();
  };
  if (!p.vec) {  // columns of C that start anywhere: element by element, sixteen lanes to a row
#pragma unroll
    for (int j = 0; j < N; j += 16) {
      put(j);
      float v[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = *reinterpret_cast<const float*>(stage + (2 * i + (lane >> 4)) * kEmitPitch + (lane & 15) * 4);
      const int64_t col = col0 + j + (lane & 15), row = row0 + (lane >> 4);
      const int rows = col < p.cols ? (int)min((int64_t)32, p.rows - row) : 0;
      TC* c = C + row * ldc + col;
      if (beta != 0.0f) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (2 * i < rows) v[i] += beta * f8_load1(c + 2 * i * ldc);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (2 * i < rows) f8_store1(c + 2 * i * ldc, v[i]);
    }
    return;
  }
  // four lanes to a row; the old values of a lane's four rows are on their way at once
  const int rows = (int)min((int64_t)32, p.rows - row0 - (lane >> 2));
#pragma unroll
  for (int j = 0; j < N; j += 16) {
    put(j);
    const int64_t col = col0 + j + piece * 4, nv = p.cols - col;
    TC* c = C + (row0 + (lane >> 2)) * ldc + col;
    if (nv >= 4) {
      float old[4][4] = {};
      if (beta != 0.0f) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (8 * i < rows) f8_load4(c + 8 * i * ldc, old[i]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float v[4];
        f8_load4(reinterpret_cast<const float*>(swap + 8 * i * kEmitPitch), v);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = beta != 0.0f ? v[e] + beta * old[i][e] : v[e];
        if (8 * i < rows) f8_store4(c + 8 * i * ldc, v);
      }
    } else {
#pragma unroll 1
      for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int e = 0; e < 3; ++e) {
          float v = *reinterpret_cast<const float*>(swap + 8 * i * kEmitPitch + 4 * e);
          if (8 * i < rows && e < nv) {
            if (beta != 0.0f) v += beta * f8_load1(c + 8 * i * ldc + e);
            f8_store1(c + 8 * i * ldc + e, v);
          }
        }
      }
    }
  }
}

// Joining the shares of a k split: the CTAs of a cluster (rank = share) have each put their sums of the same 128 x TBN tile
// into their shared memory (f8_put_share), the index that is contiguous in C contiguous there too; each CTA adds all shares, in the
// order of their rank, for its part of the other index, four numbers at a time and all ranks' numbers on their way at once
// (one after the other, their latency made up most of a 1024^3 product: 21 us, now 5.9).  All threads of all CTAs of the cluster call this; the
// 32 EW threads with worker >= 0 (numbered) add and write, unless their waits have run out (ok, the same in a warp).  PERMUTE: row r of the tile is row kept_row(r) of C.
constexpr int kMaxSplit = 8;  // 2, 4 or 8 CTAs
struct F8Split {
  int s;          // CTAs to a tile
  double clocks;  // estimate of the product's time
};
// tiles, stages of a tile's k range, clocks of a stage, clocks of a join of two, CTAs that an SM holds; defined in f8_gemm.cu
F8Split f8_split_for(int64_t tiles, int stages, double stage, double join, int resident);
__host__ __device__ constexpr int share_pitch(int inner) { return inner + 4; }  // 16-byte pieces of consecutive lines in different banks
__host__ __device__ constexpr int share_bytes(int tbn) { return 4 * (tbn * share_pitch(128) > 128 * share_pitch(tbn) ? tbn * share_pitch(128) : 128 * share_pitch(tbn)); }
__device__ __forceinline__ int kept_row(int i) { return (i & ~3) | ((i & 1) << 1) | ((i >> 1) & 1); }

// N consecutive columns from `col` of row `row` of the tile
template <bool COLS_CONTIG, int TBN, int N>
__device__ __forceinline__ void f8_put_share(void* tile, int row, int col, const float* acc) {
  float* t = static_cast<float*>(tile);
  if constexpr (COLS_CONTIG) {
#pragma unroll
    for (int j = 0; j < N; j += 4)
      *reinterpret_cast<float4*>(t + row * share_pitch(TBN) + col + j) = make_float4(acc[j], acc[j + 1], acc[j + 2], acc[j + 3]);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) t[(col + j) * share_pitch(128) + row] = acc[j];
  }
}

template <typename TC, bool COLS_CONTIG, int TBN, int EW, bool PERMUTE, int S>
__device__ __forceinline__ void f8_add_shares(const F8Out& p, void* tile, int share, int worker, int64_t row0, int64_t col0) {
  constexpr int INNER = COLS_CONTIG ? TBN : 128, OUTER = COLS_CONTIG ? 128 : TBN, PER = OUTER / S;
  constexpr int PIECES = PER * (INNER / 4), WORKERS = 32 * EW, U = (PIECES + WORKERS - 1) / WORKERS;
  uint32_t base[S];
#pragma unroll
  for (int q = 0; q < S; ++q) base[q] = cluster_map_shared(smem_u32(tile), (uint32_t)q);
  float x[U][S][4];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = worker + u * WORKERS;
    const uint32_t at = (uint32_t)((share * PER + i / (INNER / 4)) * share_pitch(INNER) + i % (INNER / 4) * 4) * 4;
#pragma unroll
    for (int q = 0; q < S; ++q)
      if (PIECES % WORKERS == 0 || i < PIECES)
        asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                     : "=f"(x[u][q][0]), "=f"(x[u][q][1]), "=f"(x[u][q][2]), "=f"(x[u][q][3])
                     : "r"(base[q] + at));
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = worker + u * WORKERS, o = share * PER + i / (INNER / 4), in = i % (INNER / 4) * 4;
    if (PIECES % WORKERS != 0 && i >= PIECES) break;
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int q = 0; q < S; ++q) v[0] += x[u][q][0], v[1] += x[u][q][1], v[2] += x[u][q][2], v[3] += x[u][q][3];
    if (PERMUTE) {
      const float t = v[1];
      v[1] = v[2], v[2] = t;
    }
    const int64_t row = row0 + (COLS_CONTIG ? o : in), col = col0 + (COLS_CONTIG ? in : o);
    const int64_t nv = COLS_CONTIG ? p.cols - col : p.rows - row;
    if (COLS_CONTIG ? row < p.rows : col < p.cols) {
      TC* c = static_cast<TC*>(p.C) + (COLS_CONTIG ? row * p.ldc + col : col * p.ldc + row);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] *= p.alpha;
      if (p.beta != 0.0f) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (e < nv) v[e] += p.beta * f8_load1(c + e);
      }
      if (!p.vec) {
        *reinterpret_cast<float4*>(static_cast<float*>(tile) + o * share_pitch(INNER) + in) = make_float4(v[0], v[1], v[2], v[3]);
      } else if (nv >= 4) {
        f8_store4(c, v);
      } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
          if (e < nv) f8_store1(c + e, v[e]);
      }
    }
  }
  if (!p.vec) {  // columns of C that start anywhere: from this CTA's own part of its own share, which no other CTA reads, lane by lane
    if (!named_barrier_all<2, WORKERS>(true)) return;
    for (int i = worker; i < PER * INNER; i += WORKERS) {
      const int o = share * PER + i / INNER, in = i % INNER;
      const int64_t row = row0 + (COLS_CONTIG ? o : in), col = col0 + (COLS_CONTIG ? in : o);
      if (row < p.rows && col < p.cols)
        f8_store1(static_cast<TC*>(p.C) + (COLS_CONTIG ? row * p.ldc + col : col * p.ldc + row), static_cast<const float*>(tile)[o * share_pitch(INNER) + in]);
    }
  }
}

// The barriers around it, and all that the warps without work do.  Where registers have been moved between warpgroups each group calls its
// part from its own branch: code they share is compiled for the smallest share.
__device__ __forceinline__ void f8_join_begin() {
  __syncwarp();
  cluster_sync_all();
}
__device__ __forceinline__ void f8_join_end() {
  __syncwarp();
  // no CTA leaves while another one reads its share; what was read has arrived, so there is nothing to release
  asm volatile("barrier.cluster.arrive.relaxed.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}
template <typename TC, bool COLS_CONTIG, int TBN, int EW, bool PERMUTE>
__device__ __forceinline__ void f8_split_join(const F8Out& p, void* tile, int splits, int share, int worker, bool ok, int64_t row0, int64_t col0) {
  f8_join_begin();
  if (worker >= 0 && !ok) {
    if (!p.vec) (void)named_barrier_all<2, 32 * EW>(false);  // where the other workers wait for this warp
  } else if (worker >= 0) {
    if (splits == 2) f8_add_shares<TC, COLS_CONTIG, TBN, EW, PERMUTE, 2>(p, tile, share, worker, row0, col0);
    else if (splits == 4) f8_add_shares<TC, COLS_CONTIG, TBN, EW, PERMUTE, 4>(p, tile, share, worker, row0, col0);
    else f8_add_shares<TC, COLS_CONTIG, TBN, EW, PERMUTE, 8>(p, tile, share, worker, row0, col0);
  }
  f8_join_end();
}

// C := beta * C, and copies of one or two operands into 16-byte aligned columns (ldd a multiple of 16 bytes); defined in f8_gemm.cu.
int f8_scale_c(int64_t m, int64_t n, float beta, void* C, int64_t ldc, int type_c, cudaStream_t st);
struct F8Copy {
  const void* src;
  int64_t ld, rows, cols;  // bytes
  void* dst;
  int64_t ldd;
};
int f8_repitch(const F8Copy* copies, int count, cudaStream_t st);

}  // namespace b2
