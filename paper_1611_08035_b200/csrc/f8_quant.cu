// Activations and weights to block-scaled 8-bit numbers: 1 byte and a 128th for the 2 or 4 that are read.  Bound by memory:
// 16384 x 8192 bf16 in 59 us (6.9 TB/s, 105 % of the copy rate), in 128 x 128 blocks 61-68 us.
#include "b2gemm.h"
#include "entry.h"
#include "f8.cuh"
#include "tcgen05.cuh"

namespace b2 {
namespace {

struct QuantArgs {
  int d;
  int64_t t;
  const void* X;
  void *Q, *S;
  int64_t ldx, ldq, lds;
};

// largest magnitudes of eight numbers as they lie in memory: bf16 in pairs, their 15 bits order like fp32's 31
__device__ __forceinline__ uint32_t raw_max(const Raw8<__nv_bfloat16>& r, uint32_t m) {
#pragma unroll
  for (int i = 0; i < 4; ++i) m = __vmaxu2(m, r.u[i] & 0x7fff7fffu);
  return m;
}
__device__ __forceinline__ uint32_t raw_max(const Raw8<float>& r, uint32_t m) {
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, r.u[i] & 0x7fffffffu);
  return m;
}
template <typename T>
__device__ __forceinline__ uint32_t join_max(uint32_t a, uint32_t b) { return sizeof(T) == 2 ? __vmaxu2(a, b) : max(a, b); }
template <typename T>
__device__ __forceinline__ uint32_t max_bits(uint32_t m) { return sizeof(T) == 2 ? max(m << 16, m & 0xffff0000u) : m; }

// One block of 128 features of one token per eight lanes, sixteen features a thread: 16-byte loads and one 16-byte store.  U blocks are
// in flight per group of lanes, one CTA's 32 U blocks following each other in memory.  Instructions are what this kernel could
// be short of (two loads of eight numbers, half as many a thread: 84 us for 16384 x 8192 bf16, for which memory needs 62), so bf16 magnitudes
// are compared in pairs.
// Q16: columns of Q on 16-byte boundaries, else on 8-byte ones.
template <typename T, int U, bool Q16>
__global__ void __launch_bounds__(256) quant_rows_kernel(const QuantArgs p, const FastDiv per_token, uint32_t total) {
  grid_started();
  grid_ready();
  const int l = threadIdx.x & 7;
  const uint32_t first = blockIdx.x * (32 * U) + (threadIdx.x >> 3);
  Raw8<T> raw[U][2];
  int64_t row[U];
  int e[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t b = first + u * 32, r = div_by(b, per_token);
    row[u] = r, e[u] = (int)(b - r * per_token.d) * kF8Block + l * 16;
    const int nv = b < total ? p.d - e[u] : 0;
    const T* x = static_cast<const T*>(p.X) + row[u] * p.ldx + e[u];
    load8(x, nv, true, raw[u][0]);
    load8(x + 8, nv - 8, true, raw[u][1]);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int nv = first + u * 32 < total ? p.d - e[u] : 0;
    uint32_t m = raw_max(raw[u][1], raw_max(raw[u][0], 0));
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) m = join_max<T>(m, __shfl_xor_sync(0xffffffffu, m, o));
    const uint32_t byte = f8_scale_byte(max_bits<T>(m));
    if (nv > 0) {
      float v[8], w[8];
      unpack8(raw[u][0], v), unpack8(raw[u][1], w);
      const uint2 a = f8_quant8(v, byte), b = f8_quant8(w, byte);
      uint8_t* q = static_cast<uint8_t*>(p.Q) + row[u] * p.ldq + e[u];
      if (Q16 && nv >= 16) {
        *reinterpret_cast<uint4*>(q) = make_uint4(a.x, a.y, b.x, b.y);
      } else {
        store8_f8(q, nv, true, a);
        store8_f8(q + 8, nv - 8, true, b);
      }
      if (l == 0) static_cast<uint8_t*>(p.S)[row[u] * p.lds + e[u] / kF8Block] = (uint8_t)byte;
    }
  }
}
// Columns that start anywhere: two blocks of a token per warp.
template <typename T, int U>
__global__ void __launch_bounds__(256) quant_rows_anywhere_kernel(const QuantArgs p, const FastDiv per_token, uint32_t total) {
  grid_started();
  grid_ready();
  using Piece = Warp256<T, false>;
  const uint32_t first = blockIdx.x * (8 * U) + (threadIdx.x >> 5);
  Raw8<T> raw[U];
  int64_t row[U];
  int at[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t b = first + u * 8, r = div_by(b, per_token);
    row[u] = r, at[u] = (int)(b - r * per_token.d) * 256;
    Piece::load(static_cast<const T*>(p.X) + row[u] * p.ldx, at[u], b < total ? p.d : 0, raw[u]);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float v[8];
    unpack8(raw[u], v);
    Piece::quantise(v, static_cast<uint8_t*>(p.Q) + row[u] * p.ldq, static_cast<uint8_t*>(p.S) + row[u] * p.lds, at[u],
                    first + u * 8 < total ? p.d : 0);
  }
}

// One 128 x 128 tile per cluster of CL CTAs, which share its rows and meet at its maximum, held in registers between that and its
// rounding: a warp has 256 of its numbers at a time, two rows.
template <typename T, bool VEC, int CL>
__global__ void __launch_bounds__(256) quant_tiles_kernel(const QuantArgs p, int64_t blocks_d) {
  grid_started();
  grid_ready();
  constexpr int N = 8 / CL;  // pieces of sixteen rows
  __shared__ uint32_t part[8], whole;
  const int64_t tile = blockIdx.x / CL, bt = tile / blocks_d, bd = tile - bt * blocks_d;
  const int row0 = CL > 1 ? (int)cluster_rank() * (kF8Block / CL) : 0;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int l = lane & 15, r = threadIdx.x >> 4;
  const int e = (int)bd * kF8Block;
  // number j of piece i: VEC: row r + 16 i, column 8 l + j; else row 16 i + 2 warp + j / 4, column 32 (j % 4) + lane
  auto row_of = [&](int i, int j) { return bt * kF8Block + row0 + (VEC ? r + 16 * i : 16 * i + 2 * warp + (j >> 2)); };
  auto col_of = [&](int j) { return e + (VEC ? 8 * l + j : 32 * (j & 3) + lane); };
  Raw8<T> raw[N];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if constexpr (VEC) {
      load8(static_cast<const T*>(p.X) + row_of(i, 0) * p.ldx + col_of(0), row_of(i, 0) < p.t ? p.d - col_of(0) : 0, true, raw[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bool in = row_of(i, j) < p.t && col_of(j) < p.d;
        if constexpr (sizeof(T) == 2) {
          const uint32_t h = in ? (uint32_t)static_cast<const uint16_t*>(p.X)[row_of(i, j) * p.ldx + col_of(j)] : 0u;
          raw[i].u[j >> 1] = j & 1 ? raw[i].u[j >> 1] | h << 16 : h;
        } else {
          raw[i].u[j] = in ? static_cast<const uint32_t*>(p.X)[row_of(i, j) * p.ldx + col_of(j)] : 0u;
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) m = raw_max(raw[i], m);
  m = __reduce_max_sync(0xffffffffu, max_bits<T>(m));
  if (lane == 0) part[warp] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, part[i]);
  if constexpr (CL > 1) {
    if (threadIdx.x == 0) whole = m;
    __syncwarp();
    cluster_sync_all();
#pragma unroll
    for (int i = 0; i < CL; ++i) {
      uint32_t v;
      asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(cluster_map_shared(smem_u32(&whole), (uint32_t)i)));
      m = max(m, v);
    }
    asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");  // no CTA leaves before the others have read its maximum
  }
  const uint32_t byte = f8_scale_byte(m);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float v[8];
    unpack8(raw[i], v);
    const uint2 q = f8_quant8(v, byte);
    uint8_t* Q = static_cast<uint8_t*>(p.Q);
    if constexpr (VEC) {
      const int64_t nv = row_of(i, 0) < p.t ? p.d - col_of(0) : 0;
      if (nv > 0) store8_f8(Q + row_of(i, 0) * p.ldq + col_of(0), nv, true, q);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (row_of(i, j) < p.t && col_of(j) < p.d) Q[row_of(i, j) * p.ldq + col_of(j)] = (uint8_t)((j < 4 ? q.x : q.y) >> (8 * (j & 3)));
    }
  }
  if (threadIdx.x == 0 && row0 == 0) static_cast<uint8_t*>(p.S)[bt * p.lds + bd] = (uint8_t)byte;
  if constexpr (CL > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
}

template <typename T>
int quant_launch(const QuantArgs& a, int block, bool vec, bool q16, cudaStream_t st) {
  const int64_t nb = blocks_of(a.d, kF8Block);
  if (block == 1) {
    constexpr int U = 2;
    const int64_t per = vec ? nb : blocks_of(a.d, 256), total = per * a.t;
    if (a.t > 0x7fffffffLL || per > 0x7fffffffLL || total > 0x7fffffffLL - 32 * U) return B2_ERR_VARIANT;  // 2^38 numbers
    const FastDiv div = fast_div((uint32_t)per);
    if (vec && q16) return launch_overlapped(quant_rows_kernel<T, U, true>, (unsigned)blocks_of(total, 32 * U), 256, st, a, div, (uint32_t)total);
    if (vec) return launch_overlapped(quant_rows_kernel<T, U, false>, (unsigned)blocks_of(total, 32 * U), 256, st, a, div, (uint32_t)total);
    return launch_overlapped(quant_rows_anywhere_kernel<T, U>, (unsigned)blocks_of(total, 8 * U), 256, st, a, div, (uint32_t)total);
  }
  const int64_t ctas = nb * blocks_of(a.t, kF8Block);
  if (ctas > 0x7fffffffLL) return B2_ERR_VARIANT;
  if (vec) return launch_overlapped(quant_tiles_kernel<T, true, 1>, (unsigned)ctas, 256, st, a, nb);
  // Few tiles of narrow accesses: four CTAs to each, so that all SMs have a share (999 x 1003 bf16 9.4 -> 5.5 us, fp32 5.8 -> 4.9).  With wide
  // accesses meeting costs more than sharing saves (1024 x 1024 bf16 2.7 us, 3.3 in clusters).
  if (ctas <= sm_count_cached()) return launch_overlapped_as(quant_tiles_kernel<T, false, 4>, dim3(4 * (unsigned)ctas), 256, 0, dim3(4), st, a, nb);
  return launch_overlapped(quant_tiles_kernel<T, false, 1>, (unsigned)ctas, 256, st, a, nb);
}

}  // namespace
}  // namespace b2

extern "C" int b2_quant_f8(int64_t d, int64_t t, int block, int type, const void* X, int64_t ldx, void* Q, int64_t ldq,
                           void* S, int64_t lds, void* cuda_stream) {
  using namespace b2;
  if (d < 0) return -1;
  if (t < 0) return -2;
  if (block != 1 && block != kF8Block) return -3;
  if (type != B2_TYPE_F32 && type != B2_TYPE_BF16) return -4;
  const bool work = d > 0 && t > 0;
  const int64_t least = d > 1 ? d : 1;
  if (work && !X) return -5;
  if (ldx < least) return -6;
  if (work && !Q) return -7;
  if (ldq < least) return -8;
  if (work && !S) return -9;
  if (lds < (d > 0 ? blocks_of(d, kF8Block) : 1)) return -10;
  if (!work) return B2_OK;
  const int es = type == B2_TYPE_BF16 ? 2 : 4;
  if (d > kMostFeatures) return B2_ERR_VARIANT;
  const QuantArgs a{(int)d, t, X, Q, S, ldx, ldq, lds};
  const bool vec = columns_aligned(X, ldx, es, 16) && columns_aligned(Q, ldq, 1, 8), q16 = columns_aligned(Q, ldq, 1, 16);
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  return type == B2_TYPE_BF16 ? quant_launch<__nv_bfloat16>(a, block, vec, q16, st) : quant_launch<float>(a, block, vec, q16, st);
}
