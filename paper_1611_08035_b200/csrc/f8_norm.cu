// Root-mean-square norm with the residual's addition and an 8-bit result, and its backward pass.
//
//   h = x + r,  rstd = 1/sqrt(mean(h^2) + eps),  y = h * rstd * w,  (q, s) = y quantised in blocks of 128 features
//   dx = rstd * (g - xh * mean(g xh)) + dh,  dw = sum_t dy xh,     g = dy w, xh = h rstd
//
// Both are bound by memory: a token is read once, kept in registers over the sum that its norm needs, and written
// once.  A thread holds groups of eight consecutive features (16 bytes of bf16), so sixteen neighbouring lanes hold
// exactly one block of 128 and its largest magnitude is four shuffles away.
#include "b2gemm.h"
#include "entry.h"
#include "f8.cuh"

namespace b2 {
namespace {

struct NormArgs {
  int64_t d, t;
  const void *X, *R, *w;
  void *H, *Q, *S;
  int64_t ldx, ldr, ldh, ldq, lds;
  float* rstd;
  float eps;
  bool vx, vr, vh, vq, vw;  // 16-byte (Q: 8-byte) alignment of every column
};

// Sum over the TPR threads of a row; the same value in each of them.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* part) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if constexpr (TPR > 32) {
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int i = 0; i < TPR / 32; ++i) v += part[i];
  }
  return v;
}

// largest bit pattern over sixteen neighbouring lanes
__device__ __forceinline__ uint32_t block_max(uint32_t b) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) b = max(b, __shfl_xor_sync(0xffffffffu, b, o));
  return b;
}

template <typename T, int TPR, int VPT>
__global__ void __launch_bounds__(TPR > 128 ? TPR : 128) norm_kernel(const NormArgs p) {
  constexpr int NT = TPR > 128 ? TPR : 128, RPC = NT / TPR;
  static_assert(RPC == 1 || TPR == 32, "rows that share a CTA meet at no barrier");
  __shared__ float part[TPR > 32 ? TPR / 32 : 1];
  const int64_t row = (int64_t)blockIdx.x * RPC + (RPC > 1 ? threadIdx.x / TPR : 0);
  const int l = RPC > 1 ? threadIdx.x % TPR : threadIdx.x;
  if (RPC > 1 && row >= p.t) return;  // whole warps
  const T* X = static_cast<const T*>(p.X) + row * p.ldx;
  const T* R = p.R ? static_cast<const T*>(p.R) + row * p.ldr : nullptr;
  T* H = p.H ? static_cast<T*>(p.H) + row * p.ldh : nullptr;
  const T* W = static_cast<const T*>(p.w);
  Raw8<T> rx[VPT], rr[VPT], rw[VPT];  // all loads first
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int64_t e = (int64_t)(l + i * TPR) * 8, nv = p.d - e;
    load8(X + e, nv, p.vx, rx[i]);
    if (R) load8(R + e, nv, p.vr, rr[i]);
  }
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int64_t e = (int64_t)(l + i * TPR) * 8, nv = p.d - e;
    load8(W + e, nv, p.vw, rw[i]);
  }
  float v[VPT][8], ss = 0.0f;
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int64_t e = (int64_t)(l + i * TPR) * 8, nv = p.d - e;
    unpack8(rx[i], v[i]);
    if (R) {
      float r[8];
      unpack8(rr[i], r);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] += r[j];
    }
    if (H) store8(H + e, nv, p.vh, v[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) ss += v[i][j] * v[i][j];
  }
  const float rstd = 1.0f / sqrtf(row_sum<TPR>(ss, part) / (float)p.d + p.eps);
  if (p.rstd && l == 0) p.rstd[row] = rstd;
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int64_t e = (int64_t)(l + i * TPR) * 8, nv = p.d - e;
    float y[8], w[8];
    uint32_t m = 0;
    unpack8(rw[i], w);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      y[j] = j < nv ? v[i][j] * rstd * w[j] : 0.0f;  // beyond the row: no 0 * inf
      m = max(m, mag_bits(y[j]));
    }
    const uint32_t byte = f8_scale_byte(block_max(m));
    if (nv > 0) {
      store8_f8(static_cast<uint8_t*>(p.Q) + row * p.ldq + e, nv, p.vq, f8_quant8(y, byte));
      if ((l & 15) == 0) static_cast<uint8_t*>(p.S)[row * p.lds + e / kF8Block] = (uint8_t)byte;
    }
  }
}

// Tokens too long for registers: the sum first, then everything else from a second reading (of L2).  h is stored in
// the second pass only, because H may be X or R.
template <typename T>
__global__ void __launch_bounds__(1024) norm_long_kernel(const NormArgs p) {
  __shared__ float part[32];
  const int64_t row = blockIdx.x;
  const T* X = static_cast<const T*>(p.X) + row * p.ldx;
  const T* R = p.R ? static_cast<const T*>(p.R) + row * p.ldr : nullptr;
  T* H = p.H ? static_cast<T*>(p.H) + row * p.ldh : nullptr;
  auto load = [&](int64_t e, float (&v)[8]) {
    load8(X + e, p.d - e, p.vx, v);
    if (R) {
      float r[8];
      load8(R + e, p.d - e, p.vr, r);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += r[j];
    }
  };
  float ss = 0.0f;
  for (int64_t e = (int64_t)threadIdx.x * 8; e < p.d; e += 8192) {
    float v[8];
    load(e, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) ss += v[j] * v[j];
  }
  const float rstd = 1.0f / sqrtf(row_sum<1024>(ss, part) / (float)p.d + p.eps);
  if (p.rstd && threadIdx.x == 0) p.rstd[row] = rstd;
  for (int64_t base = 0; base < p.d; base += 8192) {  // the same trips for every lane: block_max is warp-wide
    const int64_t e = base + (int64_t)threadIdx.x * 8, nv = p.d - e;
    float y[8], w[8];
    uint32_t m = 0;
    load(e, y);
    load8(static_cast<const T*>(p.w) + e, nv, p.vw, w);
    if (H) store8(H + e, nv, p.vh, y);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      y[j] = j < nv ? y[j] * rstd * w[j] : 0.0f;
      m = max(m, mag_bits(y[j]));
    }
    const uint32_t byte = f8_scale_byte(block_max(m));
    if (nv > 0) {
      store8_f8(static_cast<uint8_t*>(p.Q) + row * p.ldq + e, nv, p.vq, f8_quant8(y, byte));
      if ((threadIdx.x & 15) == 0) static_cast<uint8_t*>(p.S)[row * p.lds + e / kF8Block] = (uint8_t)byte;
    }
  }
}

template <typename T>
int norm_launch(const NormArgs& a, cudaStream_t st) {
  const int64_t chunks = blocks_of(a.d, 8);
  if (a.t > 0x7fffffffLL) return B2_ERR_VARIANT;
  const unsigned t = (unsigned)a.t, t4 = (unsigned)blocks_of(a.t, 4);
  if (a.t <= 2 * sm_count_cached() && chunks > 32 && chunks <= 1024) {
    // few tokens: one group of eight per thread, the shortest chain from the load to the store
    if (chunks <= 128) norm_kernel<T, 128, 1><<<t, 128, 0, st>>>(a);
    else if (chunks <= 256) norm_kernel<T, 256, 1><<<t, 256, 0, st>>>(a);
    else if (chunks <= 512) norm_kernel<T, 512, 1><<<t, 512, 0, st>>>(a);
    else norm_kernel<T, 1024, 1><<<t, 1024, 0, st>>>(a);
  } else if (chunks <= 32) norm_kernel<T, 32, 1><<<t4, 128, 0, st>>>(a);
  else if (chunks <= 64) norm_kernel<T, 32, 2><<<t4, 128, 0, st>>>(a);
  else if (chunks <= 128) norm_kernel<T, 32, 4><<<t4, 128, 0, st>>>(a);
  else if (chunks <= 256) norm_kernel<T, 128, 2><<<t, 128, 0, st>>>(a);
  else if (chunks <= 512) norm_kernel<T, 128, 4><<<t, 128, 0, st>>>(a);
  else if (chunks <= 1024) norm_kernel<T, 256, 4><<<t, 256, 0, st>>>(a);
  else if (chunks <= 2048) norm_kernel<T, 512, 4><<<t, 512, 0, st>>>(a);
  else norm_long_kernel<T><<<t, 1024, 0, st>>>(a);
  return cudaGetLastError() == cudaSuccess ? B2_OK : B2_ERR_LAUNCH;
}

// ---- backward -------------------------------------------------------------------------------------------
struct NormBwdArgs {
  int64_t d, t;
  const void *DY, *H, *w, *DH;
  void* DX;
  int64_t lddy, ldh, lddh, lddx;
  const float* rstd;
  float* partial;  // [gridDim.x][d]
  bool vy, vh, vr, vx, vw;
};

// A CTA walks over the tokens cta, cta + grid, ...; a thread owns the same features of each of them, so that its share of
// dw stays in registers until the end and leaves as one row of partial sums.
template <typename T, int NT, int VPT>
__global__ void __launch_bounds__(NT) norm_bwd_kernel(const NormBwdArgs p) {
  __shared__ float part[2][NT / 32];
  const int l = threadIdx.x;
  float dw[VPT][8];
  Raw8<T> rw[VPT], ry[VPT], rh[VPT], rg[VPT];
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int64_t e = (int64_t)(l + i * NT) * 8, nv = row < p.t ? p.d - e : 0;
      load8(static_cast<const T*>(p.DY) + row * p.lddy + e, nv, p.vy, ry[i]);
      load8(static_cast<const T*>(p.H) + row * p.ldh + e, nv, p.vh, rh[i]);
      if (p.DH) load8(static_cast<const T*>(p.DH) + row * p.lddh + e, nv, p.vr, rg[i]);
    }
  };
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int64_t e = (int64_t)(l + i * NT) * 8;
    load8(static_cast<const T*>(p.w) + e, p.d - e, p.vw, rw[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) dw[i][j] = 0.0f;
  }
  int parity = 0;
  fetch(blockIdx.x);
  for (int64_t row = blockIdx.x; row < p.t; row += gridDim.x, parity ^= 1) {
    const float rstd = p.rstd[row];
    Raw8<T> cy[VPT], ch[VPT], cg[VPT];
    float dot = 0.0f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      cy[i] = ry[i], ch[i] = rh[i], cg[i] = rg[i];
      float dy[8], xh[8], w[8];
      unpack8(cy[i], dy), unpack8(ch[i], xh), unpack8(rw[i], w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        xh[j] *= rstd;
        dot += dy[j] * w[j] * xh[j];
        dw[i][j] += dy[j] * xh[j];
      }
    }
    fetch(row + gridDim.x);  // on its way while this token's sum is taken
    const float mean = row_sum<NT>(dot, part[parity]) / (float)p.d;  // two arrays in turn: one barrier a token
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int64_t e = (int64_t)(l + i * NT) * 8, nv = p.d - e;
      float dx[8], dy[8], xh[8], w[8], dh[8];
      unpack8(cy[i], dy), unpack8(ch[i], xh), unpack8(rw[i], w);
      if (p.DH) unpack8(cg[i], dh);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        dx[j] = rstd * (dy[j] * w[j] - xh[j] * rstd * mean);
        if (p.DH) dx[j] += dh[j];
      }
      store8(static_cast<T*>(p.DX) + row * p.lddx + e, nv, p.vx, dx);
    }
  }
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int64_t e = (int64_t)(l + i * NT) * 8;
    store8(p.partial + (int64_t)blockIdx.x * p.d + e, p.d - e, (p.d & 3) == 0, dw[i]);
  }
}

// Tokens too long for registers: dx from two readings of a token ...
template <typename T>
__global__ void __launch_bounds__(1024) norm_bwd_long_kernel(const NormBwdArgs p) {
  __shared__ float part[32];
  const int64_t row = blockIdx.x;
  const T* DY = static_cast<const T*>(p.DY) + row * p.lddy;
  const T* H = static_cast<const T*>(p.H) + row * p.ldh;
  const T* W = static_cast<const T*>(p.w);
  const float rstd = p.rstd[row];
  float dot = 0.0f;
  for (int64_t e = (int64_t)threadIdx.x * 8; e < p.d; e += 8192) {
    float dy[8], h[8], w[8];
    load8(DY + e, p.d - e, p.vy, dy);
    load8(H + e, p.d - e, p.vh, h);
    load8(W + e, p.d - e, p.vw, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) dot += dy[j] * w[j] * (h[j] * rstd);
  }
  const float mean = row_sum<1024>(dot, part) / (float)p.d;
  for (int64_t e = (int64_t)threadIdx.x * 8; e < p.d; e += 8192) {
    const int64_t nv = p.d - e;
    float dy[8], h[8], w[8], dh[8];
    load8(DY + e, nv, p.vy, dy);
    load8(H + e, nv, p.vh, h);
    load8(W + e, nv, p.vw, w);
    if (p.DH) load8(static_cast<const T*>(p.DH) + row * p.lddh + e, nv, p.vr, dh);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      dy[j] = rstd * (dy[j] * w[j] - (h[j] * rstd) * mean);
      if (p.DH) dy[j] += dh[j];
    }
    store8(static_cast<T*>(p.DX) + row * p.lddx + e, nv, p.vx, dy);
  }
}
// ... and dw, before dx may overwrite dy or h, with a thread for every feature.
template <typename T>
__global__ void __launch_bounds__(256) norm_bwd_long_dw_kernel(const NormBwdArgs p) {
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (e >= p.d) return;
  float s = 0.0f;
  for (int64_t row = blockIdx.y; row < p.t; row += gridDim.y)
    s += (float)static_cast<const T*>(p.DY)[row * p.lddy + e] * ((float)static_cast<const T*>(p.H)[row * p.ldh + e] * p.rstd[row]);
  p.partial[(int64_t)blockIdx.y * p.d + e] = s;
}

// dw[e] = sum over the rows of partial sums, always in the same order.
__global__ void __launch_bounds__(512) norm_bwd_sum_kernel(const float* partial, int64_t rows, int64_t d, float* dw) {
  __shared__ float part[16][33];
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
  const int64_t e = (int64_t)blockIdx.x * 32 + x;
  float s = 0.0f;
  if (e < d)
    for (int64_t r = y; r < rows; r += 16) s += partial[r * d + e];
  part[y][x] = s;
  __syncthreads();
  if (y == 0 && e < d) {
    s = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) s += part[i][x];
    dw[e] = s;
  }
}

constexpr int64_t kBwdLongest = 2048;  // groups of eight of the longest token held in registers

// rows of partial sums: CTAs of the backward kernel
int64_t bwd_rows(int64_t d, int64_t t) {
  const int64_t chunks = blocks_of(d, 8), sms = sm_count_cached();
  int64_t rows;
  if (chunks > kBwdLongest) rows = 16;
  else rows = sms * (chunks <= 256 ? 4 : chunks <= 1024 ? 2 : 1);
  const int64_t most = blocks_of(t, 4);
  return rows < most ? rows : most;
}

template <typename T>
int norm_bwd_launch(const NormBwdArgs& a, float* dw, cudaStream_t st) {
  const int64_t chunks = blocks_of(a.d, 8), rows = bwd_rows(a.d, a.t);
  if (a.t > 0x7fffffffLL || a.d > 0x7fffffffLL) return B2_ERR_VARIANT;
  const unsigned g = (unsigned)rows;
  if (rows > 0) {
    if (chunks <= 128) norm_bwd_kernel<T, 128, 1><<<g, 128, 0, st>>>(a);
    else if (chunks <= 256) norm_bwd_kernel<T, 128, 2><<<g, 128, 0, st>>>(a);
    else if (chunks <= 512) norm_bwd_kernel<T, 256, 2><<<g, 256, 0, st>>>(a);
    else if (chunks <= 1024) norm_bwd_kernel<T, 512, 2><<<g, 512, 0, st>>>(a);
    else if (chunks <= kBwdLongest) norm_bwd_kernel<T, 512, 4><<<g, 512, 0, st>>>(a);
    else {
      norm_bwd_long_dw_kernel<T><<<dim3((unsigned)blocks_of(a.d, 256), g), 256, 0, st>>>(a);
      norm_bwd_long_kernel<T><<<(unsigned)a.t, 1024, 0, st>>>(a);
    }
  }
  norm_bwd_sum_kernel<<<(unsigned)blocks_of(a.d, 32), 512, 0, st>>>(a.partial, rows, a.d, dw);
  return cudaGetLastError() == cudaSuccess ? B2_OK : B2_ERR_LAUNCH;
}

bool type_ok(int type) { return type == B2_TYPE_F32 || type == B2_TYPE_BF16; }

}  // namespace
}  // namespace b2

extern "C" int b2_rmsnorm_f8(int64_t d, int64_t t, int type, const void* X, int64_t ldx, const void* R, int64_t ldr,
                             const void* w, float eps, void* H, int64_t ldh, void* Q, int64_t ldq, void* S, int64_t lds,
                             float* rstd, void* cuda_stream) {
  using namespace b2;
  if (d < 0) return -1;
  if (t < 0) return -2;
  if (!type_ok(type)) return -3;
  const bool work = d > 0 && t > 0;
  const int64_t least = d > 1 ? d : 1, nb = d > 0 ? blocks_of(d, kF8Block) : 1;
  if (work && !X) return -4;
  if (ldx < least) return -5;
  if (R && ldr < least) return -7;
  if (work && !w) return -8;
  if (!(eps >= 0.0f)) return -9;
  if (H && ldh < least) return -11;
  if (work && !Q) return -12;
  if (ldq < least) return -13;
  if (work && !S) return -14;
  if (lds < nb) return -15;
  if (!work) return B2_OK;
  const int es = type == B2_TYPE_BF16 ? 2 : 4;
  const NormArgs a{d, t, X, R, w, H, Q, S, ldx, ldr, ldh, ldq, lds, rstd, eps, columns_aligned(X, ldx, es, 16),
                   columns_aligned(R, ldr, es, 16), columns_aligned(H, ldh, es, 16), columns_aligned(Q, ldq, 1, 8),
                   columns_aligned(w, 0, es, 16)};
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  return type == B2_TYPE_BF16 ? norm_launch<__nv_bfloat16>(a, st) : norm_launch<float>(a, st);
}

extern "C" size_t b2_rmsnorm_backward_workspace_bytes(int64_t d, int64_t t) {
  if (d <= 0 || t <= 0) return 0;
  return b2::round_up((size_t)b2::bwd_rows(d, t) * (size_t)d * sizeof(float), 256);
}

extern "C" int b2_rmsnorm_backward(int64_t d, int64_t t, int type, const void* DY, int64_t lddy, const void* H, int64_t ldh,
                                   const float* rstd, const void* w, const void* DH, int64_t lddh, void* DX, int64_t lddx,
                                   float* dw, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  using namespace b2;
  if (d < 0) return -1;
  if (t < 0) return -2;
  if (!type_ok(type)) return -3;
  const bool work = d > 0 && t > 0;
  const int64_t least = d > 1 ? d : 1;
  if (work && !DY) return -4;
  if (lddy < least) return -5;
  if (work && !H) return -6;
  if (ldh < least) return -7;
  if (work && !rstd) return -8;
  if (work && !w) return -9;
  if (DH && lddh < least) return -11;
  if (work && !DX) return -12;
  if (lddx < least) return -13;
  if (d > 0 && !dw) return -14;
  if (d == 0) return B2_OK;
  const size_t need = b2_rmsnorm_backward_workspace_bytes(d, t);
  if (need && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0 || workspace_bytes < need)) return B2_ERR_WORKSPACE;
  const int es = type == B2_TYPE_BF16 ? 2 : 4;
  const NormBwdArgs a{d, t, DY, H, w, DH, DX, lddy, ldh, lddh, lddx, rstd, static_cast<float*>(workspace),
                      columns_aligned(DY, lddy, es, 16), columns_aligned(H, ldh, es, 16), columns_aligned(DH, lddh, es, 16),
                      columns_aligned(DX, lddx, es, 16), columns_aligned(w, 0, es, 16)};
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  return type == B2_TYPE_BF16 ? norm_bwd_launch<__nv_bfloat16>(a, dw, st) : norm_bwd_launch<float>(a, dw, st);
}
