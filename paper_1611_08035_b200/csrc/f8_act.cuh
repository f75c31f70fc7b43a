// The end of the 8-bit products with an epilogue (b2_gemm_f8_act): from the sums in registers or in a split's shares,
//
//   z = alpha * sum + bias,  c = act(z) + r        or, gradient form,        c = alpha * sum * act'(Z) + r
//
// with Z, C stored as they are and (Q, S) = c quantised, each where it is wanted.  All of it in fp32 from the unrounded sum; every result is rounded once, when
// it is stored, so that Q does not depend on C's type.
//
// A feature is an index of C that is contiguous, a token the other one.  Where results leave in whole tiles a thread holds 64 or 128
// consecutive features of a token, so that the largest magnitude of a block of 128 is at most one exchange away, and matrices pass through a warp's
// staging rows in both directions: the thread that owns a token's row computes, the lanes together read and write whole pieces of rows.
#pragma once
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
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t row = row0 + 8 * i + (lane >> 2);
      if (row < rows) {
        const uint4 q = *reinterpret_cast<const uint4*>(from + 8 * i * kEmitPitch);
        if (nv >= PIECE) {
          *reinterpret_cast<uint4*>(m + row * ld + c) = q;
        } else {
          const Bits* b = reinterpret_cast<const Bits*>(from + 8 * i * kEmitPitch);
          for (int e = 0; e < nv; ++e) m[row * ld + c + e] = b[e];
        }
      }
    }
  } else {  // columns that start anywhere: neighbouring lanes, neighbouring elements
#pragma unroll 4
    for (int i = 0; i < W; ++i) {
      const int r = W < 32 ? 2 * i + lane / L : i / D, e = W < 32 ? lane % L : i % D * 32 + lane;
      const int64_t row = row0 + r, c = col + e;
      if (row < rows && c < cols) m[row * ld + c] = *reinterpret_cast<const Bits*>(stage + r * kEmitPitch + e * (int)sizeof(T));
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
  constexpr int W = act_width<T>(), PIECE = 16 / (int)sizeof(T), L = W < 32 ? W : 32, D = W < 32 ? 1 : W / 32;  // lanes to a row, turns to a row
  const int lane = threadIdx.x & 31;
  const Bits* m = static_cast<const Bits*>(M);
  const unsigned char* own = stage + lane * kEmitPitch;
  __syncwarp();
  if (vec) {
    const int64_t c = col + (lane & 3) * PIECE, nv = p.cols - c;
    unsigned char* to = stage + (lane >> 2) * kEmitPitch + (lane & 3) * 16;
    uint4 q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t row = row0 + 8 * i + (lane >> 2);
      q[i] = make_uint4(0, 0, 0, 0);
      if (row < p.rows && nv >= PIECE) q[i] = *reinterpret_cast<const uint4*>(m + row * ld + c);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4*>(to + 8 * i * kEmitPitch) = q[i];
    if (nv > 0 && nv < PIECE) {
      for (int i = 0; i < 4; ++i) {
        const int64_t row = row0 + 8 * i + (lane >> 2);
        for (int e = 0; row < p.rows && e < nv; ++e) reinterpret_cast<Bits*>(to + 8 * i * kEmitPitch)[e] = m[row * ld + c + e];
      }
    }
  } else {
#pragma unroll 8
    for (int i = 0; i < W; ++i) {
      const int r = W < 32 ? 2 * i + lane / L : i / D, e = W < 32 ? lane % L : i % D * 32 + lane;
      const int64_t row = row0 + r, c = col + e;
      *reinterpret_cast<Bits*>(stage + r * kEmitPitch + e * (int)sizeof(T)) = row < p.rows && c < p.cols ? m[row * ld + c] : (Bits)0;
    }
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
#pragma unroll
    for (int j = 0; j < G; ++j) v[j] = col + j < p.cols ? v[j] : 0.0f;  // a block's largest magnitude is that of the matrix's own numbers
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
// A thread with whole blocks (the kernels on pairs of CTAs).
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

// ---- tiles whose rows are the features (decoding: few tokens) ---------------------------------------------------------
// One feature of N tokens a lane, four warps to a block of 128 features; `swap`: 2 x 64 x 4 words.
constexpr int kActColumnSwapBytes = 2 * 64 * 4 * 4;
template <typename TC, int N>
__device__ __forceinline__ bool act_emit_columns(const F8ActOut& p, int64_t row, int64_t col0, float* acc, uint32_t* swap, int quad, int round) {
  constexpr int G = 16;
  const bool in = row < p.rows;
  const float b = p.bias && in ? p.bias[row] : 0.0f;
#pragma unroll 1
  for (int c = 0; c < N; c += G) {
    const int64_t col = col0 + c;
    const int nv = in ? (int)max((int64_t)0, min((int64_t)G, p.cols - col)) : 0;
    float v[G], old[G];
#pragma unroll
    for (int j = 0; j < G; ++j) v[j] = p.alpha * acc[j] + b;
    if (p.gradient) {
#pragma unroll
      for (int j = 0; j < G; ++j) old[j] = j < nv ? f8_load1(static_cast<const TC*>(p.Zin) + row + (col + j) * p.ldz) : 0.0f;
      act_slopes<G>(p.act, v, old);
    } else {
      if (p.Z) {
#pragma unroll
        for (int j = 0; j < G; ++j)
          if (j < nv) f8_store1(static_cast<TC*>(p.Z) + row + (col + j) * p.ldz, v[j]);
      }
      act_values<G>(p.act, v);
    }
    if (p.R) {
#pragma unroll
      for (int j = 0; j < G; ++j) old[j] = j < nv ? f8_load1(static_cast<const TC*>(p.R) + row + (col + j) * p.ldr) : 0.0f;
#pragma unroll
      for (int j = 0; j < G; ++j) v[j] += old[j];
    }
    if (p.C) {
#pragma unroll
      for (int j = 0; j < G; ++j)
        if (j < nv) f8_store1(static_cast<TC*>(p.C) + row + (col + j) * p.ldc, v[j]);
    }
#pragma unroll
    for (int j = 0; j < N - G; ++j) acc[j] = acc[j + G];
#pragma unroll
    for (int j = 0; j < G; ++j) acc[N - G + j] = j < nv ? v[j] : 0.0f;
  }
  if (!p.Q) return true;
  swap += (round & 1) * 256;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const uint32_t m = __reduce_max_sync(0xffffffffu, mag_bits(acc[j]));
    if ((threadIdx.x & 31) == (j & 31)) swap[4 * j + quad] = m;
  }
  if (!named_barrier_all<3, 128>(true)) return false;
  const int nv = (int)min((int64_t)N, p.cols - col0);
  uint8_t* q = p.Q + row + col0 * p.ldq;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const uint4 w = *reinterpret_cast<const uint4*>(swap + 4 * j);
    const uint32_t byte = f8_scale_byte(max(max(w.x, w.y), max(w.z, w.w)));
    const uint32_t e = byte == kScaleNan ? 0x7fu : f8_pack4(acc[j] * f8_inv_scale(byte), 0.0f, 0.0f, 0.0f) & 255u;
    if (in && j < nv) {
      q[j * p.ldq] = (uint8_t)e;
      if ((row & (kF8Block - 1)) == 0) p.S[(col0 + j) * p.lds + row / kF8Block] = (uint8_t)byte;
    }
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

}  // namespace b2
