// Activations and weights to block-scaled 8-bit numbers: 1 byte and a 128th for the 2 or 4 that are read.
#include "b2gemm.h"
#include "entry.h"
#include "f8.cuh"

namespace b2 {
namespace {

struct QuantArgs {
  int64_t d, t;
  const void* X;
  void *Q, *S;
  int64_t ldx, ldq, lds;
  bool vx, vq;
};

// One block of 128 features of one token per sixteen lanes, eight features a thread.  U blocks are in flight per group of
// lanes, one CTA's 16 U blocks following each other in memory.
template <typename T, int U>
__global__ void __launch_bounds__(256) quant_rows_kernel(const QuantArgs p, const FastDiv per_token, uint32_t total) {
  const int l = threadIdx.x & 15;
  const uint32_t first = blockIdx.x * (16 * U) + (threadIdx.x >> 4);
  Raw8<T> raw[U];
  int64_t row[U], e[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t b = first + u * 16, r = div_by(b, per_token);
    row[u] = r, e[u] = (int64_t)(b - r * per_token.d) * kF8Block + l * 8;
    load8(static_cast<const T*>(p.X) + row[u] * p.ldx + e[u], b < total ? p.d - e[u] : 0, p.vx, raw[u]);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t nv = first + u * 16 < total ? p.d - e[u] : 0;
    float v[8];
    unpack8(raw[u], v);
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, mag_bits(v[j]));
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    const uint32_t byte = f8_scale_byte(m);
    if (nv > 0) {
      store8_f8(static_cast<uint8_t*>(p.Q) + row[u] * p.ldq + e[u], nv, p.vq, f8_quant8(v, byte));
      if (l == 0) static_cast<uint8_t*>(p.S)[row[u] * p.lds + e[u] / kF8Block] = (uint8_t)byte;
    }
  }
}

// One 128 x 128 tile per CTA, held in registers between its maximum and its rounding.
template <typename T>
__global__ void __launch_bounds__(256) quant_tiles_kernel(const QuantArgs p, int64_t blocks_d) {
  __shared__ uint32_t part[8];
  const int64_t bt = blockIdx.x / blocks_d, bd = blockIdx.x - bt * blocks_d;
  const int l = threadIdx.x & 15, r = threadIdx.x >> 4;
  const int64_t e = bd * kF8Block + l * 8;
  Raw8<T> raw[8];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t row = bt * kF8Block + r + 16 * i;
    load8(static_cast<const T*>(p.X) + row * p.ldx + e, row < p.t ? p.d - e : 0, p.vx, raw[i]);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float v[8];
    unpack8(raw[i], v);
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, mag_bits(v[j]));
  }
  m = __reduce_max_sync(0xffffffffu, m);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, part[i]);
  const uint32_t byte = f8_scale_byte(m);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t row = bt * kF8Block + r + 16 * i, nv = row < p.t ? p.d - e : 0;
    float v[8];
    unpack8(raw[i], v);
    if (nv > 0) store8_f8(static_cast<uint8_t*>(p.Q) + row * p.ldq + e, nv, p.vq, f8_quant8(v, byte));
  }
  if (threadIdx.x == 0) static_cast<uint8_t*>(p.S)[bt * p.lds + bd] = (uint8_t)byte;
}

template <typename T>
int quant_launch(const QuantArgs& a, int block, cudaStream_t st) {
  const int64_t nb = blocks_of(a.d, kF8Block);
  if (block == 1) {
    constexpr int U = 4;
    const int64_t total = nb * a.t;
    if (a.t > 0x7fffffffLL || total > 0x7fffffffLL - 16 * U) return B2_ERR_VARIANT;  // 2^38 numbers
    quant_rows_kernel<T, U><<<(unsigned)blocks_of(total, 16 * U), 256, 0, st>>>(a, fast_div((uint32_t)nb), (uint32_t)total);
  } else {
    const int64_t ctas = nb * blocks_of(a.t, kF8Block);
    if (ctas > 0x7fffffffLL) return B2_ERR_VARIANT;
    quant_tiles_kernel<T><<<(unsigned)ctas, 256, 0, st>>>(a, nb);
  }
  return cudaGetLastError() == cudaSuccess ? B2_OK : B2_ERR_LAUNCH;
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
  const QuantArgs a{d, t, X, Q, S, ldx, ldq, lds, columns_aligned(X, ldx, es, 16), columns_aligned(Q, ldq, 1, 8)};
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  return type == B2_TYPE_BF16 ? quant_launch<__nv_bfloat16>(a, block, st) : quant_launch<float>(a, block, st);
}
