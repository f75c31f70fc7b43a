// The end of the 8-bit products with an epilogue (b2_gemm_f8_act): from the sums in registers or in a split's shares,
//
//   z = alpha * sum + bias,  c = act(z) + r        or, gradient form,        c = alpha * sum * act'(Z) + r
//
// with Z, C stored as they are and (Q, S) = c quantised, each where it is wanted.  All of it in fp32 from the unrounded sum; every result is rounded once, when
// it is stored: Q from the unrounded c, not from C.
//
// A feature is an index of C that is contiguous, a token the other one.  Where results leave in whole tiles a thread holds 64 or 128
// consecutive features of a token, so that the largest magnitude of a block of 128 is at most one exchange away, and matrices pass through a warp's
// staging rows in both directions: the thread that owns a token's row computes, the lanes together read and write whole pieces of rows.
#pragma once
#include <cuda.h>

#include "act.cuh"
#include "f8_out.cuh"

namespace b2 {

struct F8ActOut {
  int64_t rows, cols;  // extents of the MMA's row and column index
  float alpha;
  int act, gradient;
  const float* bias;
  const void* Zin;  // gradient form
  void *Z, *C;      // Z: the forward form's
  const void* R;
  int64_t ldz, ldr, ldc;
  int vz, vr, vc, vb;  // columns are 16-byte aligned (vb: the bias is)
  uint8_t *Q, *S;
  int64_t ldq, lds;
  int vq;
};

// ---- matrices between memory and the rows that a warp's lanes own -------------------------------------------------------
// 64 bytes of each of 32 rows at a time; W numbers.
template <typename T>
__host__ __device__ constexpr int act_width() { return 64 / (int)sizeof(T); }

template <typename T>
__device__ __forceinline__ uint4 act_pack16(const float* v) {  // 16 bytes
  if constexpr (sizeof(T) == 2) return make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
  else return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}
template <typename T>
__device__ __forceinline__ void act_unpack16(const uint4& q, float* v) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    else v[i] = __uint_as_float(w[i]);
  }
}
template <typename T>
struct ActBits {
  using type = uint32_t;
};
template <>
struct ActBits<__nv_bfloat16> {
  using type = uint16_t;
};
template <>
struct ActBits<uint8_t> {
  using type = uint8_t;
};

// What lies in the staging rows leaves for M[row][col ..], rows row0 .. row0 + 31.
template <typename T>
__device__ __forceinline__ void act_rows_out(T* M, int64_t ld, bool vec, int64_t rows, int64_t cols, int64_t row0, int64_t col, const unsigned char* stage) {
  using Bits = typename ActBits<T>::type;
  constexpr int W = act_width<T>(), PIECE = 16 / (int)sizeof(T), L = W < 32 ? W : 32, D = W < 32 ? 1 : W / 32;  // lanes to a row, turns to a row
  const int lane = threadIdx.x & 31;
  Bits* m = reinterpret_cast<Bits*>(M);
  if (vec) {
    const int64_t c = col + (lane & 3) * PIECE, nv = cols - c;
    const unsigned char* from = stage + (lane >> 2) * kEmitPitch + (lane & 3) * 16;
    uint4 q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = *reinterpret_cast<const uint4*>(from + 8 * i * kEmitPitch);
    Bits* to = m + (row0 + (lane >> 2)) * ld + c;
    if (row0 + 32 <= rows && col + W <= cols) {
#pragma unroll
      for (int i = 0; i < 4; ++i, to += 8 * ld) *reinterpret_cast<uint4*>(to) = q[i];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i, to += 8 * ld) {
        const bool here = row0 + 8 * i + (lane >> 2) < rows;
        if (here && nv >= PIECE) {
          *reinterpret_cast<uint4*>(to) = q[i];
        } else if (here && nv > 0) {
          const uint32_t w[4] = {q[i].x, q[i].y, q[i].z, q[i].w};
#pragma unroll
          for (int e = 0; e < PIECE - 1; ++e)
            if (e < nv) to[e] = (Bits)(w[e * (int)sizeof(T) / 4] >> (e * (int)sizeof(T) % 4 * 8));
        }
      }
    }
  } else {  // columns that start anywhere: neighbouring lanes, neighbouring elements.  Tested one by one everywhere, bf16 4097 x 4096 x 1024 took 228 us, now 108
    const int r0 = lane / L, e0 = lane % L;
    Bits* to = m + (row0 + r0) * ld + col + e0;
    const unsigned char* from = stage + r0 * kEmitPitch + e0 * (int)sizeof(T);
    if (row0 + 32 <= rows && col + W <= cols) {
#pragma unroll 16
      for (int i = 0; i < W; ++i) {
        to[i % D * 32] = *reinterpret_cast<const Bits*>(from + i / D * (32 / L) * kEmitPitch + i % D * 32 * (int)sizeof(T));
        if (i % D == D - 1) to += 32 / L * ld;
      }
    } else {
#pragma unroll 4
      for (int i = 0; i < W; ++i) {
        const int64_t row = row0 + r0 + i / D * (32 / L), c = col + e0 + i % D * 32;
        if (row < rows && c < cols) m[row * ld + c] = *reinterpret_cast<const Bits*>(from + i / D * (32 / L) * kEmitPitch + i % D * 32 * (int)sizeof(T));
      }
    }
  }
}
template <typename T>
__device__ __forceinline__ void act_put(void* M, int64_t ld, bool vec, const F8ActOut& p, int64_t row0, int64_t col, const float* v, unsigned char* stage) {
  unsigned char* own = stage + (threadIdx.x & 31) * kEmitPitch;
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4*>(own + 16 * i) = act_pack16<T>(v + i * (16 / (int)sizeof(T)));
  __syncwarp();
  act_rows_out<T>(static_cast<T*>(M), ld, vec, p.rows, p.cols, row0, col, stage);
}
// The other way; numbers outside the matrix are 0.
template <typename T>
__device__ __forceinline__ void act_get(const void* M, int64_t ld, bool vec, const F8ActOut& p, int64_t row0, int64_t col, float* v, unsigned char* stage) {
  using Bits = typename ActBits<T>::type;
  constexpr int W = act_width<T>(), PIECE = 16 / (int)sizeof(T), L = W < 32 ? W : 32, RW = 32 / L;  // lanes to a row, rows of a turn
  const int lane = threadIdx.x & 31;
  const Bits* m = static_cast<const Bits*>(M);
  const unsigned char* own = stage + lane * kEmitPitch;
  __syncwarp();
  if (vec) {
    const int64_t c = col + (lane & 3) * PIECE, nv = p.cols - c;
    unsigned char* to = stage + (lane >> 2) * kEmitPitch + (lane & 3) * 16;
    const Bits* from = m + (row0 + (lane >> 2)) * ld + c;
    uint4 q[4];
    if (row0 + 32 <= p.rows && col + W <= p.cols) {
#pragma unroll
      for (int i = 0; i < 4; ++i, from += 8 * ld) q[i] = *reinterpret_cast<const uint4*>(from);
#pragma unroll
      for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4*>(to + 8 * i * kEmitPitch) = q[i];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        q[i] = make_uint4(0, 0, 0, 0);
        if (row0 + 8 * i + (lane >> 2) < p.rows && nv >= PIECE) q[i] = *reinterpret_cast<const uint4*>(from + 8 * i * ld);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4*>(to + 8 * i * kEmitPitch) = q[i];
      if (nv > 0 && nv < PIECE) {  // all on their way together
        const int here = (int)min((int64_t)32, p.rows - row0) - (lane >> 2);
        Bits x[4][PIECE - 1];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < PIECE - 1; ++e) x[i][e] = e < nv && 8 * i < here ? from[8 * i * ld + e] : (Bits)0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < PIECE - 1; ++e) reinterpret_cast<Bits*>(to + 8 * i * kEmitPitch)[e] = x[i][e];
      }
    }
  } else {
    const int r0 = lane / L;
    const int64_t c = col + lane % L;
    const Bits* from = m + (row0 + r0) * ld + c;
    unsigned char* to = stage + r0 * kEmitPitch + lane % L * (int)sizeof(T);
    const int here = c < p.cols ? (int)min((int64_t)32, p.rows - row0) : 0;  // rows
#pragma unroll 16
    for (int i = 0; i < W; ++i, from += RW * ld) *reinterpret_cast<Bits*>(to + i * RW * kEmitPitch) = r0 + i * RW < here ? *from : (Bits)0;
  }
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 4; ++i) act_unpack16<T>(*reinterpret_cast<const uint4*>(own + 16 * i), v + i * PIECE);
}

// R, and in the gradient form Z, on their way to L2 while the tile is computed (rows of a warp's part of the tile, `count` columns).
template <typename TC>
__device__ __forceinline__ void f8_prefetch(const F8ActOut& p, bool, int64_t row0, int lines, int64_t first, int count) {
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const TC* m = static_cast<const TC*>(which ? p.R : p.Zin);
    const int64_t ld = which ? p.ldr : p.ldz;
    if (!m) continue;
    for (int i = threadIdx.x & 31; i < lines; i += 32)
      for (int e = 0; e < count; e += 128 / (int)sizeof(TC))
        if (row0 + i < p.rows && first + e < p.cols) asm volatile("prefetch.global.L2 [%0];" ::"l"(m + (row0 + i) * ld + first + e));
  }
}

// The bias of `count` features from `first` on.
__device__ __forceinline__ void act_prefetch_bias(const F8ActOut& p, int64_t first, int count, int64_t features) {
  const int i = (threadIdx.x & 31) * 32;
  if (p.bias && i < count && first + i < features) asm volatile("prefetch.global.L1 [%0];" ::"l"(p.bias + first + i));
}
// What a warp of a small tile will read, on its way while the tile is computed: its rows (COLS_CONTIG) or columns, `count` numbers each; of a split's, the part that this CTA
// will add up.
template <typename TC, bool COLS_CONTIG, int TBN>
__device__ __forceinline__ void act_prefetch_small(const F8ActOut& p, int64_t row0, int64_t col0, int ew, int workers, int splits, int share) {
  constexpr int INNER = COLS_CONTIG ? TBN : 128, OUTER = COLS_CONTIG ? 128 : TBN;
  const int64_t feature0 = COLS_CONTIG ? col0 : row0, token0 = COLS_CONTIG ? row0 : col0, features = COLS_CONTIG ? p.cols : p.rows, tokens = COLS_CONTIG ? p.rows : p.cols;
  if (ew == 0) act_prefetch_bias(p, feature0, INNER, features);
  const int per = OUTER / splits;
  for (int o = ew * 32 + (threadIdx.x & 31); o < per; o += 32 * workers) {
    const int64_t token = token0 + share * per + o;
    if (token >= tokens) break;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      const TC* m = static_cast<const TC*>(which ? p.R : p.Zin);
      if (!m) continue;
      m += token * (which ? p.ldr : p.ldz) + feature0;
      for (int e = 0; e < INNER && feature0 + e < features; e += 128 / (int)sizeof(TC)) asm volatile("prefetch.global.L2 [%0];" ::"l"(m + e));
    }
  }
}

// ---- tiles whose columns are the features ------------------------------------------------------------------------------
// N consecutive features of 32 consecutive tokens (row0 + lane); acc holds the results c afterwards, 0 beyond the matrix.  32 columns a turn of a
// loop that is not unrolled, through which the accumulators move: unrolled, with each function's code in all four places, it is 300 KB of instructions.
template <typename TC, int N>
__device__ __forceinline__ void act_emit_rows(const F8ActOut& p, int64_t row0, int64_t col0, float* acc, unsigned char* stage) {
  constexpr int G = 32, W = act_width<TC>();
#pragma unroll 1
  for (int c = 0; c < N; c += G) {
    const int64_t col = col0 + c;
    float v[G];
#pragma unroll
    for (int j = 0; j < G; ++j) v[j] = p.alpha * acc[j];
    if (col < p.cols) {
      if (p.gradient) {
        float z[G];
#pragma unroll
        for (int h = 0; h < G; h += W) act_get<TC>(p.Zin, p.ldz, p.vz, p, row0, col + h, z + h, stage);
        act_slopes<G>(p.act, v, z);
      } else {
        if (p.bias) {
          const float* b = p.bias + col;
          if (p.vb && col + G <= p.cols) {
#pragma unroll
            for (int j = 0; j < G; j += 4) {
              const float4 f = *reinterpret_cast<const float4*>(b + j);
              v[j] += f.x, v[j + 1] += f.y, v[j + 2] += f.z, v[j + 3] += f.w;
            }
          } else {
#pragma unroll
            for (int j = 0; j < G; ++j) v[j] += col + j < p.cols ? b[j] : 0.0f;
          }
        }
        if (p.Z) {
#pragma unroll
          for (int h = 0; h < G; h += W) act_put<TC>(p.Z, p.ldz, p.vz, p, row0, col + h, v + h, stage);
        }
        act_values<G>(p.act, v);
      }
      if (p.R) {
        float r[G];
#pragma unroll
        for (int h = 0; h < G; h += W) act_get<TC>(p.R, p.ldr, p.vr, p, row0, col + h, r + h, stage);
#pragma unroll
        for (int j = 0; j < G; ++j) v[j] += r[j];
      }
      if (p.C) {
#pragma unroll
        for (int h = 0; h < G; h += W) act_put<TC>(p.C, p.ldc, p.vc, p, row0, col + h, v + h, stage);
      }
    }
    if (col + G > p.cols) {  // a block's largest magnitude is that of the matrix's own numbers
#pragma unroll
      for (int j = 0; j < G; ++j) v[j] = col + j < p.cols ? v[j] : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < N - G; ++j) acc[j] = acc[j + G];
#pragma unroll
    for (int j = 0; j < G; ++j) acc[N - G + j] = v[j];
  }
}
template <int N>
__device__ __forceinline__ uint32_t act_amax(const float* acc) {
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < N; ++j) m = max(m, mag_bits(acc[j]));
  return m;
}
// N results of each lane's row as e4m3 numbers under the block's largest magnitude; the thread with the block's first features writes its scale.
template <int N>
__device__ __forceinline__ void act_quantise_rows(const F8ActOut& p, int64_t row0, int64_t col0, const float* acc, uint32_t amax, bool writes_scale, unsigned char* stage) {
  if (col0 >= p.cols) return;
  const int lane = threadIdx.x & 31;
  const uint32_t byte = f8_scale_byte(amax);
  if (writes_scale && row0 + lane < p.rows) p.S[(row0 + lane) * p.lds + col0 / kF8Block] = (uint8_t)byte;
#pragma unroll
  for (int j = 0; j < N; j += 64) {
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float y[2][8];
#pragma unroll
      for (int e = 0; e < 16; ++e) y[e >> 3][e & 7] = acc[j + 16 * i + e];
      const uint2 a = f8_quant8(y[0], byte), b = f8_quant8(y[1], byte);
      *reinterpret_cast<uint4*>(stage + lane * kEmitPitch + 16 * i) = make_uint4(a.x, a.y, b.x, b.y);
    }
    __syncwarp();
    act_rows_out<uint8_t>(p.Q, p.ldq, p.vq, p.rows, p.cols, row0, col0 + j, stage);
  }
}
// A thread with whole blocks: the kernels on pairs of CTAs, where a matrix's columns start anywhere.
template <typename TC, int N>
__device__ __forceinline__ void f8_emit_staged(const F8ActOut& p, int64_t row0, int64_t col0, float* acc, unsigned char* stage) {
  static_assert(N == kF8Block, "a thread holds one block of a token");
  act_emit_rows<TC, N>(p, row0, col0, acc, stage);
  if (p.Q) act_quantise_rows<N>(p, row0, col0, acc, act_amax<N>(acc), true, stage);
}
// Half a block a thread: warps w and w + 4 have the two halves of the same tokens.  `swap`: 2 x 8 x 32 words, used in turn (`round`), so that a warp that comes to
// the next tile does not overwrite what its partner has yet to read.  All eight warps meet at the barrier; false where one of them has given up.
constexpr int kActSwapBytes = 2 * 8 * 32 * 4;
template <typename TC>
__device__ __forceinline__ bool act_emit_halves(const F8ActOut& p, int64_t row0, int64_t col0, float* acc, unsigned char* stage, uint32_t* swap, int ew, int round) {
  constexpr int N = kF8Block / 2;
  act_emit_rows<TC, N>(p, row0, col0, acc, stage);
  if (!p.Q) return true;
  const int lane = threadIdx.x & 31;
  swap += (round & 1) * 256;
  uint32_t m = act_amax<N>(acc);
  swap[ew * 32 + lane] = m;
  if (!named_barrier_all<3, 256>(true)) return false;
  m = max(m, swap[(ew ^ 4) * 32 + lane]);
  act_quantise_rows<N>(p, row0, col0, acc, m, ew < 4, stage);
  return true;
}

// ---- tiles of pairs of CTAs --------------------------------------------------------------------------------------------------
// A thread has a whole block, 128 consecutive features of one token.  Two warps a scheduler have little to hide latencies behind, so that what they do is kept short and
// nothing in it waits for memory: matrices pass through pieces of shared memory, 32 bytes of 32 rows each, swizzled so that the rows' owners read and write them
// without conflicts.  Results leave by TMA (edges are the tensor maps', for columns of whole 16 bytes); what is read comes by cp.async, a piece ahead; the bias lies in shared memory.
// Clocks of a tile for a warp, two on a scheduler: alpha and bias 2700, gelu 5500 (4100 of it the unit for exp and 1/x), its slope 8000 (measured before it was as exact where it is small, which is 2 % of the kernel's time), a result 3000, what is read 3000, the 8-bit
// result 2300.  Not kept, all 8192 x 4096 x 256: staged both ways as act_emit_rows does it (with bias, gelu, Z and Q 107 us, now 60); R read by its rows' owners, 64 bytes a row (78 us, now 54); R and
// Z by TMA, whose small loads wait behind the operands' large ones (1200 clocks a piece; gradient of gelu with C and Q 96 us, now 82); sixteen warps with 64 columns and 96 registers (86; and
// the scales' and the issuing warps', left with 56 and 40, hold the tensor core up: C alone 16384 x 8192 x 4096 387 -> 481 us).
constexpr int kActPiece = 32 * 32;
constexpr int kActBias = kF8Block * 4;
// GRADIENT: the form with a kernel of its own, so that either's instructions are few.
template <int PIECES, bool GRADIENT>
struct F8ActTiles : F8ActOut {
  static constexpr int WARP_BYTES = PIECES * kActPiece + kActBias;
  CUtensorMap mz, mc, mq;  // of Z, C and Q where they are written
};
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, const void* smem, int c_inner, int c_outer) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"(reinterpret_cast<uint64_t>(map)), "r"(c_inner), "r"(c_outer),
               "r"(smem_u32(smem))
               : "memory");
}
// A warp's pieces: the first for what is read, the others for results.
template <int PIECES>
struct ActPieces {
  unsigned char* at;  // the pieces, then the bias

  __device__ __forceinline__ static unsigned char* mine(unsigned char* piece, int row, int half) { return piece + row * 32 + ((row >> 2 & 1) ^ half) * 16; }
  // COUNT times 32 bytes of each lane's row to (col, row0 ..), `step` columns apart, as far as they lie before `end`
  template <int COUNT>
  __device__ __forceinline__ void put(const CUtensorMap* map, int col, int step, int end, int row0, const uint4* w) {
    const int lane = threadIdx.x & 31;
    unsigned char* s = at + (PIECES - COUNT) * kActPiece;
    if (lane == 0) bulk_wait_read_all();
    __syncwarp();
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
      *reinterpret_cast<uint4*>(mine(s + i * kActPiece, lane, 0)) = w[2 * i];
      *reinterpret_cast<uint4*>(mine(s + i * kActPiece, lane, 1)) = w[2 * i + 1];
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) {
#pragma unroll
      for (int i = 0; i < COUNT; ++i)
        if (col + i * step < end) tma_store_2d(map, s + i * kActPiece, col + i * step, row0);
      bulk_commit();
    }
  }
  // Where this lane's shares of what is read begin, two rows of 16 bytes a piece, at the tile's first column.
  const unsigned char *base = nullptr, *from = nullptr, *from16 = nullptr;
  int left = 0, left16 = 0;  // bytes of those rows
  template <typename TC>
  __device__ __forceinline__ void read_from(const void* M, int64_t ld, const F8ActOut& p, int64_t row0, int64_t col0) {
    const int lane = threadIdx.x & 31, r = lane >> 1;
    base = static_cast<const unsigned char*>(M);
    from = reinterpret_cast<const unsigned char*>(static_cast<const TC*>(M) + (row0 + r) * ld + col0) + (lane & 1) * 16;
    from16 = from + 16 * ld * (int64_t)sizeof(TC);
    const int bytes = (int)min((int64_t)kF8Block, p.cols - col0) * (int)sizeof(TC) - (lane & 1) * 16;
    left = row0 + r < p.rows ? bytes : 0, left16 = row0 + r + 16 < p.rows ? bytes : 0;
  }
  // the piece to read is filled with 32 bytes of every row, `at_byte` of the tile; 0 beyond the matrix
  __device__ __forceinline__ void ask(int at_byte) {
    const int lane = threadIdx.x & 31;
    unsigned char* to = mine(at, lane >> 1, lane & 1);  // sixteen rows on the swizzle is the same
    const int a = min(16, left - at_byte), b = min(16, left16 - at_byte);
    cp_async_zfill<16>(to, a > 0 ? from + at_byte : base, max(a, 0));
    cp_async_zfill<16>(to + 512, b > 0 ? from16 + at_byte : base, max(b, 0));
    cp_async_commit();
  }
  // 32 bytes of each lane's row, once they have arrived
  __device__ __forceinline__ void take(uint4& a, uint4& b) const {
    const int lane = threadIdx.x & 31;
    unsigned char* piece = at;
    cp_async_wait<0>();
    __syncwarp();
    a = *reinterpret_cast<const uint4*>(mine(piece, lane, 0));
    b = *reinterpret_cast<const uint4*>(mine(piece, lane, 1));
    __syncwarp();
  }
  __device__ __forceinline__ float* bias() const { return reinterpret_cast<float*>(at + PIECES * kActPiece); }
  // no CTA leaves before its results have
  __device__ __forceinline__ void drain() const {
    if ((threadIdx.x & 31) == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    cp_async_wait<0>();
  }
};
// Before the sums are waited for: the bias of the tile's features, 0 beyond the matrix and where there is none, and the first pieces of what is read.
template <typename TC, int PIECES, bool GRADIENT>
__device__ __forceinline__ void act_begin_tile(const F8ActTiles<PIECES, GRADIENT>& p, int64_t row0, int64_t col0, ActPieces<PIECES>& pieces) {
  if (row0 >= p.rows || col0 >= p.cols) return;  // the warp's part of an edge tile lies outside
  const int64_t col = col0 + 4 * (threadIdx.x & 31);
  float4 b = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  if (!GRADIENT && p.bias) {
    if (p.vb && col + 4 <= p.cols) {
      b = *reinterpret_cast<const float4*>(p.bias + col);
    } else {
      if (col < p.cols) b.x = p.bias[col];
      if (col + 1 < p.cols) b.y = p.bias[col + 1];
      if (col + 2 < p.cols) b.z = p.bias[col + 2];
      if (col + 3 < p.cols) b.w = p.bias[col + 3];
    }
  }
  if (GRADIENT || p.R) {
    cp_async_wait<0>();  // an edge tile before this one leaves a piece that it did not take
    pieces.template read_from<TC>(GRADIENT ? p.Zin : p.R, GRADIENT ? p.ldz : p.ldr, p, row0, col0);
    pieces.ask(0);
  }
  if (!GRADIENT) {
    __syncwarp();
    reinterpret_cast<float4*>(pieces.bias())[threadIdx.x & 31] = b;
    __syncwarp();
  }
}
template <typename TC, int PIECES, bool GRADIENT>
__device__ __forceinline__ void act_emit_tile(const F8ActTiles<PIECES, GRADIENT>& p, int64_t row0, int64_t col0, float* acc, ActPieces<PIECES>& pieces) {
  constexpr int G = 32, N = kF8Block, H = 16 / (int)sizeof(TC), W = 2 * H;  // numbers of 16 bytes, of a row of a piece
  if (row0 >= p.rows || col0 >= p.cols) return;
  const int64_t row = row0 + (threadIdx.x & 31);
  const int end = (int)min((int64_t)N, p.cols - col0);
  const bool reads = GRADIENT || p.R;
  auto put = [&](const CUtensorMap* map, int c, const float* v) {
    if (PIECES == 2) {
#pragma unroll
      for (int j = 0; j < G; j += W) {
        const uint4 w[2] = {act_pack16<TC>(v + j), act_pack16<TC>(v + j + H)};
        if (c + j < end) pieces.template put<1>(map, (int)col0 + c + j, W, (int)col0 + end, (int)row0, w);
      }
    } else {
#pragma unroll
      for (int j = 0; j < G; j += 2 * W) {
        const uint4 w[4] = {act_pack16<TC>(v + j), act_pack16<TC>(v + j + H), act_pack16<TC>(v + j + W), act_pack16<TC>(v + j + W + H)};
        if (c + j < end) pieces.template put<2>(map, (int)col0 + c + j, W, (int)col0 + end, (int)row0, w);
      }
    }
  };
  // 32 columns a turn of a loop that is not unrolled, through which the accumulators move: fetching instructions costs as much as they do (64 a turn: gradient of gelu with C and
  // Q 102 us instead of 88)
#pragma unroll 1
  for (int c = 0; c < N; c += G) {
    float v[G];
    if (!GRADIENT && p.bias) {
      const float4* b = reinterpret_cast<const float4*>(pieces.bias()) + c / 4;
#pragma unroll
      for (int j = 0; j < G; j += 4) {
        const float4 f = b[j / 4];
        const Two x = fma2({acc[j], acc[j + 1]}, both(p.alpha), {f.x, f.y}), y = fma2({acc[j + 2], acc[j + 3]}, both(p.alpha), {f.z, f.w});
        v[j] = x.a, v[j + 1] = x.b, v[j + 2] = y.a, v[j + 3] = y.b;
      }
    } else {
#pragma unroll
      for (int j = 0; j < G; j += 2) {
        const Two x = mul2({acc[j], acc[j + 1]}, both(p.alpha));
        v[j] = x.a, v[j + 1] = x.b;
      }
    }
    if (c < end) {
      if (!GRADIENT && p.Z) put(&p.mz, c, v);
      if (reads) {
#pragma unroll
        for (int j = 0; j < G; j += W) {
          uint4 x, y;
          pieces.take(x, y);
          if (c + j + W < N) pieces.ask((c + j + W) * (int)sizeof(TC));
          float m[W];
          act_unpack16<TC>(x, m);
          act_unpack16<TC>(y, m + H);
          if constexpr (GRADIENT) {
            act_slopes<W>(p.act, v + j, m);
            if (p.R) {  // read in the middle of the work
              const TC* r = static_cast<const TC*>(p.R) + row * p.ldr + col0 + c + j;
#pragma unroll
              for (int e = 0; e < W; ++e) m[e] = row < p.rows && c + j + e < end ? f8_load1(r + e) : 0.0f;
            }
          } else {
            act_values<W>(p.act, v + j);
          }
          if (p.R) {
#pragma unroll
            for (int e = 0; e < W; e += 2) {
              const Two t = add2({v[j + e], v[j + e + 1]}, {m[e], m[e + 1]});
              v[j + e] = t.a, v[j + e + 1] = t.b;
            }
          }
        }
      } else if constexpr (!GRADIENT) {
        act_values<G>(p.act, v);
      }
      if (p.C) put(&p.mc, c, v);
    }
#pragma unroll
    for (int j = 0; j < N - G; ++j) acc[j] = acc[j + G];
#pragma unroll
    for (int j = 0; j < G; ++j) acc[N - G + j] = v[j];
  }
  if (!p.Q) return;
  float most[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int j = 0; j < N; ++j) most[j & 3] = larger_nan(most[j & 3], fabsf(acc[j]));
  const uint32_t byte = f8_scale_byte(__float_as_uint(larger_nan(larger_nan(most[0], most[1]), larger_nan(most[2], most[3]))));
  if (row < p.rows) p.S[row * p.lds + col0 / kF8Block] = (uint8_t)byte;
  const float inv = byte == kScaleNan ? 0.0f : f8_inv_scale(byte);
  constexpr int Q = PIECES - 1 < 2 ? 1 : 2;  // pieces of 32 numbers at a time
#pragma unroll
  for (int j = 0; j < N; j += 32 * Q) {
    uint4 q[2 * Q];
#pragma unroll
    for (int i = 0; i < 2 * Q; ++i) {
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float* a = acc + j + 16 * i + 4 * e;
        const Two x = mul2({a[0], a[1]}, both(inv)), y = mul2({a[2], a[3]}, both(inv));
        w[e] = byte == kScaleNan ? 0x7f7f7f7fu : f8_pack4(x.a, x.b, y.a, y.b);
      }
      q[i] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    if (j < end) pieces.template put<Q>(&p.mq, (int)col0 + j, 32, (int)col0 + end, (int)row0, q);
  }
}

// ---- tiles whose rows are the features (decoding: few tokens) ---------------------------------------------------------
// One feature of N tokens a lane with its bias b, four warps to a block of 128 features; `swap`: 2 x 64 x 4 words.
constexpr int kActColumnSwapBytes = 2 * 64 * 4 * 4;
// A CTA comes here once, with nothing of this code in its instruction cache, and every line of it is waited for: hence few columns a turn.
template <typename TC, int N>
__device__ __forceinline__ bool act_emit_columns(const F8ActOut& p, int64_t row, int64_t col0, float* acc, float b, uint32_t* swap, int quad, int round) {
  constexpr int G = N <= 16 ? 4 : 8;
  const bool in = row < p.rows;
  const int cols = (int)min((int64_t)N, p.cols - col0), mine = in ? cols : 0;
  swap += (round & 1) * 256;
#pragma unroll 1
  for (int c = 0; c < N; c += G) {
    float v[G];
#pragma unroll
    for (int j = 0; j < G; ++j) v[j] = acc[j];
    if (c < cols) {
      const int64_t col = col0 + c;
      float old[G];
#pragma unroll
      for (int j = 0; j < G; ++j) v[j] = fmaf(p.alpha, v[j], b);
      if (p.gradient) {
#pragma unroll
        for (int j = 0; j < G; ++j) old[j] = c + j < mine ? f8_load1(static_cast<const TC*>(p.Zin) + row + (col + j) * p.ldz) : 0.0f;
        act_slopes<G>(p.act, v, old);
      } else {
        if (p.Z) {
#pragma unroll
          for (int j = 0; j < G; ++j)
            if (c + j < mine) f8_store1(static_cast<TC*>(p.Z) + row + (col + j) * p.ldz, v[j]);
        }
        act_values<G>(p.act, v);
      }
      if (p.R) {
#pragma unroll
        for (int j = 0; j < G; ++j) old[j] = c + j < mine ? f8_load1(static_cast<const TC*>(p.R) + row + (col + j) * p.ldr) : 0.0f;
#pragma unroll
        for (int j = 0; j < G; ++j) v[j] += old[j];
      }
      if (p.C) {
#pragma unroll
        for (int j = 0; j < G; ++j)
          if (c + j < mine) f8_store1(static_cast<TC*>(p.C) + row + (col + j) * p.ldc, v[j]);
      }
      if (p.Q) {
#pragma unroll
        for (int j = 0; j < G; ++j) {
          v[j] = c + j < mine ? v[j] : 0.0f;
          const uint32_t m = __reduce_max_sync(0xffffffffu, mag_bits(v[j]));
          if ((threadIdx.x & 31) == 0) swap[4 * (c + j) + quad] = m;
        }
      }
    }
#pragma unroll
    for (int j = 0; j < N - G; ++j) acc[j] = acc[j + G];
#pragma unroll
    for (int j = 0; j < G; ++j) acc[N - G + j] = v[j];
  }
  if (!p.Q) return true;
  if (!named_barrier_all<3, 128>(true)) return false;
  uint8_t* q = p.Q + row + col0 * p.ldq;
  uint8_t* s = (row & (kF8Block - 1)) == 0 && in ? p.S + col0 * p.lds + row / kF8Block : nullptr;
#pragma unroll 1
  for (int c = 0; c < cols; c += G) {
#pragma unroll
    for (int j = 0; j < G; ++j) {
      const uint4 w = *reinterpret_cast<const uint4*>(swap + 4 * (c + j));
      const uint32_t byte = f8_scale_byte(max(max(w.x, w.y), max(w.z, w.w)));
      const uint32_t e = byte == kScaleNan ? 0x7fu : f8_pack4(acc[j] * f8_inv_scale(byte), 0.0f, 0.0f, 0.0f) & 255u;
      if (c + j < mine) q[(c + j) * p.ldq] = (uint8_t)e;
      if (s && c + j < cols) s[(c + j) * p.lds] = (uint8_t)byte;
    }
#pragma unroll
    for (int j = 0; j < N - G; ++j) acc[j] = acc[j + G];
  }
  return true;
}

// ---- single numbers: the join of a split, and products without terms ----------------------------------------------------
// Four features of one token, at + e * step.  Loads come first.
template <typename TC>
__device__ __forceinline__ void act_finish4(const F8ActOut& p, int64_t token, int64_t tokens, int64_t at, int step, int64_t features, float (&v)[4]) {
  bool in[4];
  float z[4] = {}, r[4] = {};
#pragma unroll
  for (int e = 0; e < 4; ++e) in[e] = token < tokens && at + e * step < features;
  auto load = [&](const void* M, int64_t ld, int vec, float (&x)[4]) {
    const TC* m = static_cast<const TC*>(M) + token * ld + at;
    if (step == 1 && vec && in[3]) {
      f8_load4(m, x);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = in[e] ? f8_load1(m + e * step) : 0.0f;
    }
  };
  auto store = [&](void* M, int64_t ld, int vec) {
    TC* m = static_cast<TC*>(M) + token * ld + at;
    if (step == 1 && vec && in[3]) {
      f8_store4(m, v);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (in[e]) f8_store1(m + e * step, v[e]);
    }
  };
  if (p.gradient) load(p.Zin, p.ldz, p.vz, z);
  if (p.R) load(p.R, p.ldr, p.vr, r);
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] *= p.alpha;
  if (p.gradient) {
    act_slopes<4>(p.act, v, z);
  } else {
    if (p.bias) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += in[e] ? p.bias[at + e * step] : 0.0f;
    }
    if (p.Z) store(p.Z, p.ldz, p.vz);
    act_values<4>(p.act, v);
  }
  if (p.R) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += r[e];
  }
  if (p.C) store(p.C, p.ldc, p.vc);
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = in[e] ? v[e] : 0.0f;
}
// A block of 128 features of one token, four to each lane of a warp.
__device__ __forceinline__ void act_quantise4(const F8ActOut& p, int64_t token, int64_t tokens, int64_t block0, int at, int step, int64_t features, const float (&v)[4]) {
  const uint32_t byte = f8_scale_byte(__reduce_max_sync(0xffffffffu, max(max(mag_bits(v[0]), mag_bits(v[1])), max(mag_bits(v[2]), mag_bits(v[3])))));
  const float inv = byte == kScaleNan ? 0.0f : f8_inv_scale(byte);
  const uint32_t w = byte == kScaleNan ? 0x7f7f7f7fu : f8_pack4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
  if (token >= tokens || block0 >= features) return;
  uint8_t* q = p.Q + token * p.ldq + block0 + at;
  if (step == 1 && p.vq && block0 + at + 4 <= features) {
    *reinterpret_cast<uint32_t*>(q) = w;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (block0 + at + e * step < features) q[e * step] = (uint8_t)(w >> (8 * e));
  }
  if ((threadIdx.x & 31) == 0) p.S[token * p.lds + block0 / kF8Block] = (uint8_t)byte;
}

// As f8_add_shares.  A warp has 128 numbers at a time: a token's 128 features, or 64 of two tokens (COLS_CONTIG, TBN 64; not where Q is wanted).  Matrices whose columns
// start anywhere: the warp's sums pass through its part of this CTA's own share, which no other CTA reads, so that neighbouring lanes have neighbours.
template <typename TC, bool COLS_CONTIG, int TBN, int EW, int S>
__device__ __forceinline__ void act_add_shares(const F8ActOut& p, void* tile, int share, int worker, int64_t row0, int64_t col0) {
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
  const bool rows_of_four = (!p.Z || p.vz) && (!p.Zin || p.vz) && (!p.R || p.vr) && (!p.C || p.vc) && (!p.Q || p.vq);
  const int64_t features = COLS_CONTIG ? p.cols : p.rows, tokens = COLS_CONTIG ? p.rows : p.cols;
  const int lane = threadIdx.x & 31;
  float sum[U][4];
#pragma unroll
  for (int u = 0; u < U; ++u) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      sum[u][e] = 0.0f;
#pragma unroll
      for (int q = 0; q < S; ++q) sum[u][e] += x[u][q][e];
    }
  }
#pragma unroll 1
  for (int i = worker; i < PIECES; i += WORKERS) {  // whole warps: PIECES is a multiple of 32.  The sums move through sum[0], as in act_emit_rows
    if ((COLS_CONTIG ? row0 : col0) + share * PER + (i - lane) / (INNER / 4) >= tokens) break;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = sum[0][e];
#pragma unroll
      for (int u = 1; u < U; ++u) sum[u - 1][e] = sum[u][e];
    }
    int o = share * PER + i / (INNER / 4), in = i % (INNER / 4) * 4;
    if (rows_of_four) {
      act_finish4<TC>(p, (COLS_CONTIG ? row0 : col0) + o, tokens, (COLS_CONTIG ? col0 : row0) + in, 1, features, v);
      if (INNER == kF8Block && p.Q) act_quantise4(p, (COLS_CONTIG ? row0 : col0) + o, tokens, COLS_CONTIG ? col0 : row0, in, 1, features, v);
    } else {
      float* t = static_cast<float*>(tile);
      *reinterpret_cast<float4*>(t + o * share_pitch(INNER) + in) = make_float4(v[0], v[1], v[2], v[3]);
      __syncwarp();
      o = share * PER + (i - lane) / (INNER / 4);  // the warp's first row
      if constexpr (INNER == kF8Block) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = t[o * share_pitch(INNER) + lane + 32 * e];
        act_finish4<TC>(p, (COLS_CONTIG ? row0 : col0) + o, tokens, (COLS_CONTIG ? col0 : row0) + lane, 32, features, v);
        if (p.Q) act_quantise4(p, (COLS_CONTIG ? row0 : col0) + o, tokens, COLS_CONTIG ? col0 : row0, lane, 32, features, v);
      } else {  // sixteen lanes to a row
        static_assert(INNER == kF8Block || INNER == 64, "rows of a warp");
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = t[(o + (lane >> 4)) * share_pitch(INNER) + (lane & 15) + 16 * e];
        act_finish4<TC>(p, row0 + o + (lane >> 4), tokens, col0 + (lane & 15), 16, features, v);
      }
    }
  }
}
template <typename TC, bool COLS_CONTIG, int TBN, int EW, bool PERMUTE>
__device__ __forceinline__ void f8_split_join(const F8ActOut& p, void* tile, int splits, int share, int worker, bool ok, int64_t row0, int64_t col0) {
  static_assert(!PERMUTE, "the weight gradient has no epilogue");
  f8_join_begin();
  if (worker >= 0 && ok) {
    if (splits == 2) act_add_shares<TC, COLS_CONTIG, TBN, EW, 2>(p, tile, share, worker, row0, col0);
    else if (splits == 4) act_add_shares<TC, COLS_CONTIG, TBN, EW, 4>(p, tile, share, worker, row0, col0);
    else act_add_shares<TC, COLS_CONTIG, TBN, EW, 8>(p, tile, share, worker, row0, col0);
  }
  f8_join_end();
}

// How the kernels on pairs of CTAs hand a tile over: shared memory of a warp, and whether it is by act_emit_tile.
template <typename OUT>
struct ActHandOver {
  static constexpr int WARP_BYTES = kEmitBytes;
  static constexpr bool TILES = false;
};
template <int PIECES, bool GRADIENT>
struct ActHandOver<F8ActTiles<PIECES, GRADIENT>> {
  static constexpr int WARP_BYTES = F8ActTiles<PIECES, GRADIENT>::WARP_BYTES;
  static constexpr bool TILES = true;
};

}  // namespace b2
