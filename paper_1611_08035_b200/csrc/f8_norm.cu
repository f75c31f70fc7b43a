// Root-mean-square norm with the residual's addition and an 8-bit result, and its backward pass.
//
//   h = x + r,  rstd = 1/sqrt(mean(h^2) + eps),  y = h * rstd * w,  (q, s) = y quantised in blocks of 128 features
//   dx = rstd * (g - xh * mean(g xh)) + dh,  dw = sum_t dy xh,     g = dy w, xh = h rstd
//
// Sizes here are tokens x features.  Both are bound by memory: a token is read once, kept in registers over the sum that its norm needs, and written once.  A
// warp holds 256 consecutive features, exactly two blocks of 128, so that their largest magnitudes never leave it.
// Measured, bf16: norm of 16384 x 8192 153 us (6.1 TB/s, 94 % of the copy rate), gradient of 16384 x 8192 181 us (5.9 TB/s); fp32: 270 us
// (6.5 TB/s) and 326 us (6.6 TB/s).  Other lengths: norm of 2560 features 5.8, of 3184 4.2, of 10240 5.5 TB/s; gradient of 2560 4.6, of
// 5120 4.4, of 7168 5.5 TB/s.  bf16 tokens that do not start on 16 bytes are read two bytes at a time: 1.8 TB/s.
#include "b2gemm.h"
#include "entry.h"
#include "f8.cuh"

namespace b2 {
namespace {

struct NormArgs {
  int d;
  int64_t t;
  const void *X, *R, *w;
  void *H, *Q, *S;
  int64_t ldx, ldr, ldh, ldq, lds;
  float* rstd;
  float eps;
};

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// Sum over a CTA of NT threads (FULL) or at most as many; the same value in each of them.
template <int NT, bool FULL>
__device__ __forceinline__ float cta_sum(float v, float* part) {
  v = warp_sum(v);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  if (!FULL && threadIdx.x < NT / 32 && threadIdx.x >= blockDim.x / 32) part[threadIdx.x] = 0.0f;  // the first warp has a lane for each missing one
  __syncthreads();
  v = 0.0f;
#pragma unroll
  for (int i = 0; i < NT / 32; ++i) v += part[i];
  return v;
}

// WARP: a warp to a token, four tokens a CTA; otherwise the CTA, whose size is the token's.  A thread holds VPT groups of eight features
// (Warp256: which eight).  FULL: the CTA has NT threads, which saves 4 % where it does (8192 x 8192 bf16 80 us, 83 with a width read at
// run time); otherwise as many warps as the token fills (16384 x 2560: 70 us with the next power of two, 51).
template <typename T, int VPT, int NT, bool WARP, bool VEC, bool FULL = true>
__global__ void __launch_bounds__(NT, NT == 512 && VPT == 4 && sizeof(T) == 2 ? 2 : 1) norm_kernel(const NormArgs p) {
  grid_started();
  grid_ready();
  using Piece = Warp256<T, VEC>;
  __shared__ float part[NT / 32];
  const int64_t row = WARP ? (int64_t)blockIdx.x * (NT / 32) + threadIdx.x / 32 : blockIdx.x;
  const int l = WARP ? threadIdx.x % 32 : threadIdx.x, width = WARP ? 32 : FULL ? NT : (int)blockDim.x;
  if (WARP && row >= p.t) return;  // whole warps
  const T* X = static_cast<const T*>(p.X) + row * p.ldx;
  const T* R = p.R ? static_cast<const T*>(p.R) + row * p.ldr : nullptr;
  T* H = p.H ? static_cast<T*>(p.H) + row * p.ldh : nullptr;
  auto first = [&](int i) { return ((l & ~31) + i * width) * 8; };
  Raw8<T> rx[VPT], rr[VPT], rw[VPT];  // all loads first
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    Piece::load(X, first(i), p.d, rx[i]);
    if (R) Piece::load(R, first(i), p.d, rr[i]);
  }
#pragma unroll
  for (int i = 0; i < VPT; ++i) Piece::load(static_cast<const T*>(p.w), first(i), p.d, rw[i]);
  float v[VPT][8], ss = 0.0f;
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    unpack8(rx[i], v[i]);
    if (R) {
      float r[8];
      unpack8(rr[i], r);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] += r[j];
    }
    if (H) Piece::store(H, first(i), p.d, v[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) ss += v[i][j] * v[i][j];
  }
  const float rstd = 1.0f / sqrtf((WARP ? warp_sum(ss) : cta_sum<NT, FULL>(ss, part)) / (float)p.d + p.eps);
  if (p.rstd && l == 0) p.rstd[row] = rstd;
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    float y[8], w[8];
    unpack8(rw[i], w);
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = Piece::index(first(i), j) < p.d ? v[i][j] * rstd * w[j] : 0.0f;  // beyond the row: no 0 * inf
    Piece::quantise(y, static_cast<uint8_t*>(p.Q) + row * p.ldq, static_cast<uint8_t*>(p.S) + row * p.lds, first(i), p.d);
  }
}

// Tokens too long for registers: the sum first, then everything else from a second reading (of L2).  h is stored in
// the second pass only, because H may be X or R.
template <typename T, bool VEC>
__global__ void __launch_bounds__(1024) norm_long_kernel(const NormArgs p) {
  grid_started();
  grid_ready();
  using Piece = Warp256<T, VEC>;
  __shared__ float part[32];
  const int64_t row = blockIdx.x;
  const T* X = static_cast<const T*>(p.X) + row * p.ldx;
  const T* R = p.R ? static_cast<const T*>(p.R) + row * p.ldr : nullptr;
  T* H = p.H ? static_cast<T*>(p.H) + row * p.ldh : nullptr;
  auto load = [&](int first, float (&v)[8]) {
    Raw8<T> a, b;
    Piece::load(X, first, p.d, a);
    if (R) Piece::load(R, first, p.d, b);
    unpack8(a, v);
    if (R) {
      float r[8];
      unpack8(b, r);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += r[j];
    }
  };
  float ss = 0.0f;
  for (int first = (int)(threadIdx.x & ~31u) * 8; first < p.d; first += 8192) {
    float v[8];
    load(first, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) ss += v[j] * v[j];
  }
  const float rstd = 1.0f / sqrtf(cta_sum<1024, true>(ss, part) / (float)p.d + p.eps);
  if (p.rstd && threadIdx.x == 0) p.rstd[row] = rstd;
  for (int first = (int)(threadIdx.x & ~31u) * 8; first < p.d; first += 8192) {  // the same for the lanes of a warp
    float y[8], w[8];
    Raw8<T> rw;
    Piece::load(static_cast<const T*>(p.w), first, p.d, rw);
    load(first, y);
    unpack8(rw, w);
    if (H) Piece::store(H, first, p.d, y);
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = Piece::index(first, j) < p.d ? y[j] * rstd * w[j] : 0.0f;
    Piece::quantise(y, static_cast<uint8_t*>(p.Q) + row * p.ldq, static_cast<uint8_t*>(p.S) + row * p.lds, first, p.d);
  }
}

template <typename T, bool VEC>
int norm_launch(const NormArgs& a, cudaStream_t st) {
  const int64_t chunks = blocks_of(a.d, 8);
  if (a.t > 0x7fffffffLL) return B2_ERR_VARIANT;
  const unsigned t = (unsigned)a.t, t4 = (unsigned)blocks_of(a.t, 4);
  int rc;
  if (a.t <= 2 * sm_count_cached() && chunks > 32 && chunks <= 1024) {
    // few tokens: one group of eight per thread, the shortest chain from the load to the store
    if (chunks <= 128) rc = launch_overlapped(norm_kernel<T, 1, 128, false, VEC>, t, 128, st, a);
    else if (chunks <= 256) rc = launch_overlapped(norm_kernel<T, 1, 256, false, VEC>, t, 256, st, a);
    else if (chunks <= 512) rc = launch_overlapped(norm_kernel<T, 1, 512, false, VEC>, t, 512, st, a);
    else rc = launch_overlapped(norm_kernel<T, 1, 1024, false, VEC>, t, 1024, st, a);
  } else if (chunks <= 32) rc = launch_overlapped(norm_kernel<T, 1, 128, true, VEC>, t4, 128, st, a);
  else if (chunks <= 64) rc = launch_overlapped(norm_kernel<T, 2, 128, true, VEC>, t4, 128, st, a);
  else if (chunks <= 128) rc = launch_overlapped(norm_kernel<T, 4, 128, true, VEC>, t4, 128, st, a);
  else if (chunks <= 2048) {
    int vpt = chunks <= 256 ? 2 : 4;  // groups of a thread: as many as leave the fewest threads without one
    auto threads = [&](int v) { return 32 * blocks_of(chunks, 32 * v); };
    for (int v = 4; v >= 2; --v)
      if (threads(v) <= 256 && threads(v) * v < threads(vpt) * vpt) vpt = v;
    const unsigned n = (unsigned)threads(vpt);
    if (vpt == 2 && n == 128) rc = launch_overlapped(norm_kernel<T, 2, 128, false, VEC>, t, n, st, a);
    else if (vpt == 2) rc = launch_overlapped(norm_kernel<T, 2, 256, false, VEC, false>, t, n, st, a);
    else if (vpt == 3) rc = launch_overlapped(norm_kernel<T, 3, 256, false, VEC, false>, t, n, st, a);
    else if (n == 128) rc = launch_overlapped(norm_kernel<T, 4, 128, false, VEC>, t, n, st, a);
    else if (n == 192) rc = launch_overlapped(norm_kernel<T, 4, 192, false, VEC>, t, n, st, a);
    else if (n == 256) rc = launch_overlapped(norm_kernel<T, 4, 256, false, VEC>, t, n, st, a);
    else if (n < 256) rc = launch_overlapped(norm_kernel<T, 4, 256, false, VEC, false>, t, n, st, a);
    else if (n == 512) rc = launch_overlapped(norm_kernel<T, 4, 512, false, VEC>, t, n, st, a);
    else rc = launch_overlapped(norm_kernel<T, 4, 512, false, VEC, false>, t, n, st, a);
  } else rc = launch_overlapped(norm_long_kernel<T, VEC>, t, 1024, st, a);
  return rc;
}

// ---- backward -------------------------------------------------------------------------------------------
struct NormBwdArgs {
  int d;
  int64_t t;
  const void *DY, *H, *w, *DH;
  void* DX;
  int64_t lddy, ldh, lddh, lddx;
  const float* rstd;
  float* partial;  // [gridDim.x][d]
};

// CTAs of a size that an SM holds: 128 registers a thread of bf16, 170 of fp32
constexpr int bwd_resident(size_t elem, int threads) {
  const int n = (elem == 2 ? 512 : 384) / threads;
  return n > 1 ? n : 1;
}
// A CTA walks over the tokens; a thread owns the same features of each of them, so that its share of dw stays in registers until the
// end and leaves as one row of partial sums.  TPR threads to a token, NT / TPR tokens at a time (one, or one to a warp).
template <typename T, int TPR, int NT, int VPT, bool VEC>
__global__ void __launch_bounds__(NT, bwd_resident(sizeof(T), NT)) norm_bwd_kernel(const NormBwdArgs p) {
  grid_started();
  grid_ready();
  using Piece = Warp256<T, VEC>;
  constexpr int RPC = NT / TPR;
  static_assert(RPC == 1 || TPR == 32, "tokens that share a CTA meet at no barrier");
  __shared__ float part[2][TPR / 32];
  const int l = RPC > 1 ? threadIdx.x % TPR : threadIdx.x, sub = RPC > 1 ? threadIdx.x / TPR : 0;
  const int64_t step = (int64_t)gridDim.x * RPC;
  auto first = [&](int i) { return ((l & ~31) + i * TPR) * 8; };
  float dw[VPT][8];
  Raw8<T> rw[VPT], ry[VPT], rh[VPT], rg[VPT];
  auto fetch = [&](int64_t row) {
    const int n = row < p.t ? p.d : 0;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      Piece::load(static_cast<const T*>(p.DY) + row * p.lddy, first(i), n, ry[i]);
      Piece::load(static_cast<const T*>(p.H) + row * p.ldh, first(i), n, rh[i]);
      if (p.DH) Piece::load(static_cast<const T*>(p.DH) + row * p.lddh, first(i), n, rg[i]);
    }
  };
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    Piece::load(static_cast<const T*>(p.w), first(i), p.d, rw[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) dw[i][j] = 0.0f;
  }
  int parity = 0;
  const int64_t begin = (int64_t)blockIdx.x * RPC + sub;
  fetch(begin);
  for (int64_t row = begin; row < p.t; row += step, parity ^= 1) {
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
    fetch(row + step);  // on its way while this token's sum is taken
    const float mean = (RPC > 1 ? warp_sum(dot) : cta_sum<TPR, true>(dot, part[parity])) / (float)p.d;  // two arrays in turn: one barrier a token
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      float dx[8], dy[8], xh[8], w[8], dh[8];
      unpack8(cy[i], dy), unpack8(ch[i], xh), unpack8(rw[i], w);
      if (p.DH) unpack8(cg[i], dh);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        dx[j] = rstd * (dy[j] * w[j] - xh[j] * rstd * mean);
        if (p.DH) dx[j] += dh[j];
      }
      Piece::store(static_cast<T*>(p.DX) + row * p.lddx, first(i), p.d, dx);
    }
  }
  if constexpr (RPC > 1) {  // the warps' shares, added in their order
    __shared__ float sums[NT / 32][VPT * 8 * 32];
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) sums[sub][(i * 8 + j) * 32 + l] = dw[i][j];
    __syncthreads();
    for (int k = threadIdx.x; k < VPT * 256; k += NT) {
      float s = 0.0f;
#pragma unroll
      for (int r = 0; r < RPC; ++r) s += sums[r][k];
      const int i = k / 256, j = k / 32 % 8, lane = k % 32;
      const int e = i * 256 + (VEC ? lane * 8 + j : j * 32 + lane);
      if (e < p.d) p.partial[(int64_t)blockIdx.x * p.d + e] = s;
    }
  } else {
    float* partial = p.partial + (int64_t)blockIdx.x * p.d;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int e = Piece::index(first(i), 0);
      if constexpr (VEC) {
        store8(partial + e, p.d - e, (p.d & 3) == 0, dw[i]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (Piece::index(first(i), j) < p.d) partial[Piece::index(first(i), j)] = dw[i][j];
      }
    }
  }
}

// dx of one token by 256 threads, for tokens of any length, in two readings of it.
template <typename T, bool VEC>
__device__ __forceinline__ void norm_bwd_token(const NormBwdArgs& p, int64_t row, float* part) {
  using Piece = Warp256<T, VEC>;
  const T* DY = static_cast<const T*>(p.DY) + row * p.lddy;
  const T* H = static_cast<const T*>(p.H) + row * p.ldh;
  const T* W = static_cast<const T*>(p.w);
  const float rstd = p.rstd[row];
  float dot = 0.0f;
  for (int first = (int)(threadIdx.x & ~31u) * 8; first < p.d; first += 2048) {
    Raw8<T> a, b, c;
    Piece::load(DY, first, p.d, a), Piece::load(H, first, p.d, b), Piece::load(W, first, p.d, c);
    float dy[8], h[8], w[8];
    unpack8(a, dy), unpack8(b, h), unpack8(c, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) dot += dy[j] * w[j] * (h[j] * rstd);
  }
  const float mean = cta_sum<256, true>(dot, part) / (float)p.d;
  for (int first = (int)(threadIdx.x & ~31u) * 8; first < p.d; first += 2048) {
    Raw8<T> a, b, c, g;
    Piece::load(DY, first, p.d, a), Piece::load(H, first, p.d, b), Piece::load(W, first, p.d, c);
    if (p.DH) Piece::load(static_cast<const T*>(p.DH) + row * p.lddh, first, p.d, g);
    float dx[8], h[8], w[8], dh[8];
    unpack8(a, dx), unpack8(b, h), unpack8(c, w);
    if (p.DH) unpack8(g, dh);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      dx[j] = rstd * (dx[j] * w[j] - (h[j] * rstd) * mean);
      if (p.DH) dx[j] += dh[j];
    }
    Piece::store(static_cast<T*>(p.DX) + row * p.lddx, first, p.d, dx);
  }
}

// Few tokens, in one launch: the first `tokens` CTAs write dx of a token each, the others dw of 64 features each, reading dy and h
// once more (from L2) instead of meeting the first ones' partial sums.  tokens is t, or 0 where dx is written over dy or h
// and a second launch has to follow (norm_bwd_token_kernel, the same arithmetic).  Tokens too long for registers go the same
// way; if there are many, CTAs (., y) take every gridDim.y-th group of 32 and leave partial sums.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) norm_bwd_few_kernel(const NormBwdArgs p, float* dw, int tokens) {
  grid_started();
  grid_ready();
  __shared__ float sums[32][65];
  if ((int)blockIdx.x < tokens) {
    norm_bwd_token<T, VEC>(p, blockIdx.x, &sums[0][0]);
    return;
  }
  const int x = threadIdx.x & 7, y = threadIdx.x >> 3;  // eight features a thread, every 32nd token
  const int e0 = ((int)blockIdx.x - tokens) * 64;
  float s[8] = {};
  auto at = [&](int j) { return e0 + (VEC ? x * 8 + j : j * 8 + x); };
#pragma unroll 4
  for (int64_t row = blockIdx.y * 32 + y; row < p.t; row += 32 * gridDim.y) {
    const T* DY = static_cast<const T*>(p.DY) + row * p.lddy;
    const T* H = static_cast<const T*>(p.H) + row * p.ldh;
    const float rstd = p.rstd[row];
    float dy[8], h[8];
    if constexpr (VEC) {
      load8(DY + at(0), p.d - at(0), true, dy), load8(H + at(0), p.d - at(0), true, h);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        dy[j] = at(j) < p.d ? (float)DY[at(j)] : 0.0f;
        h[j] = at(j) < p.d ? (float)H[at(j)] : 0.0f;
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] += dy[j] * (h[j] * rstd);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) sums[y][VEC ? x * 8 + j : j * 8 + x] = s[j];
  __syncthreads();
  if (threadIdx.x < 64 && e0 + threadIdx.x < p.d) {
    float v = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; ++i) v += sums[i][threadIdx.x];
    (gridDim.y > 1 ? p.partial + (int64_t)blockIdx.y * p.d : dw)[e0 + threadIdx.x] = v;
  }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(256) norm_bwd_token_kernel(const NormBwdArgs p) {
  grid_started();
  grid_ready();
  __shared__ float part[8];
  norm_bwd_token<T, VEC>(p, blockIdx.x, part);
}

// dw[e] = sum over the rows of partial sums, always in the same order.
__global__ void __launch_bounds__(1024) norm_bwd_sum_kernel(const float* partial, int64_t rows, int64_t d, float* dw) {
  grid_started();
  grid_ready();
  __shared__ float part[32][33];
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
  const int64_t e = (int64_t)blockIdx.x * 32 + x;
  float s = 0.0f;
  if (e < d) {
#pragma unroll 4
    for (int64_t r = y; r < rows; r += 32) s += partial[r * d + e];
  }
  part[y][x] = s;
  __syncthreads();
  if (y == 0 && e < d) {
    s = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; ++i) s += part[i][x];
    dw[e] = s;
  }
}

constexpr int64_t kBwdLongest = 1024;  // groups of eight of the longest token held in registers

// threads of a CTA that holds a token of more than 64 groups, two groups a thread.  An SM holds as many CTAs of 192 as of 256; three warps
// are slower than four in bf16 (16384 x 1536: 47 us against 42), not in fp32 (4096 x 1152: 19 against 25).
int bwd_threads(int64_t chunks, size_t elem) {
  const int n = 32 * (int)blocks_of(chunks, 64);
  return n == 96 && elem == 2 ? 128 : n <= 160 ? n : n <= 256 ? 256 : 512;
}
// A group a thread for up to 128 groups where there are too few tokens for an SM to hold all the CTAs it could (1001 x 1003 fp32: 8.3 us
// against 9.7; 16384 x 896 bf16 would take 33 against 28).
bool bwd_short(int64_t chunks, int64_t t) { return chunks > 64 && chunks <= 128 && t < 12 * (int64_t)sm_count_cached(); }

// rows of partial sums: CTAs of the backward kernel
int64_t bwd_rows(int64_t d, int64_t t, size_t elem) {
  const int64_t chunks = blocks_of(d, 8), sms = sm_count_cached();
  if (chunks > kBwdLongest) {
    const int64_t splits = blocks_of(t, 256);
    return splits < 16 ? splits : 16;
  }
  const int64_t rows = sms * (bwd_short(chunks, t) ? 6 : bwd_resident(elem, chunks <= 64 ? 256 : bwd_threads(chunks, elem)));
  const int64_t most = blocks_of(t, chunks <= 64 ? 32 : chunks <= 256 ? 2 : 4);  // a few tokens each, as many CTAs as fit at a time
  return rows < most ? rows : most;
}

// One launch where launches are what takes the time (bf16: 8 x 4096 3.0 us, 7.6 with two; 300 x 4096 6.1 and 8.7), two where the walk over
// the tokens does (1024 x 4096: 21 us, 14 with two; fp32 1001 x 1003: 23 us and 11).
bool bwd_few(int64_t d, int64_t t) { return t <= 384 && t * d <= (int64_t)3 << 19; }

template <typename T, bool VEC>
int norm_bwd_launch(const NormBwdArgs& a, float* dw, cudaStream_t st) {
  const int64_t chunks = blocks_of(a.d, 8), rows = bwd_rows(a.d, a.t, sizeof(T));
  if (a.t > 0x7fffffffLL) return B2_ERR_VARIANT;
  int rc = B2_OK;
  if (a.t > 0 && (bwd_few(a.d, a.t) || chunks > kBwdLongest)) {
    const bool few = bwd_few(a.d, a.t), apart = !few || a.DX == a.DY || a.DX == a.H;
    const int tokens = apart ? 0 : (int)a.t;
    const unsigned splits = few ? 1 : (unsigned)rows;
    rc = launch_overlapped(norm_bwd_few_kernel<T, VEC>, dim3((unsigned)(tokens + blocks_of(a.d, 64)), splits), 256, st, a, dw, tokens);
    if (!rc && splits > 1) rc = launch_overlapped(norm_bwd_sum_kernel, (unsigned)blocks_of(a.d, 32), 1024, st, a.partial, rows, (int64_t)a.d, dw);
    if (!rc && apart) rc = launch_overlapped(norm_bwd_token_kernel<T, VEC>, (unsigned)a.t, 256, st, a);
    return rc;
  }
  const unsigned g = (unsigned)rows;
  if (rows > 0) {
    if (chunks <= 32) rc = launch_overlapped(norm_bwd_kernel<T, 32, 256, 1, VEC>, g, 256, st, a);
    else if (chunks <= 64) rc = launch_overlapped(norm_bwd_kernel<T, 32, 256, 2, VEC>, g, 256, st, a);
    else if (bwd_short(chunks, a.t)) rc = launch_overlapped(norm_bwd_kernel<T, 128, 128, 1, VEC>, g, 128, st, a);
    else switch (bwd_threads(chunks, sizeof(T))) {
      case 64: rc = launch_overlapped(norm_bwd_kernel<T, 64, 64, 2, VEC>, g, 64, st, a); break;
      case 96: rc = launch_overlapped(norm_bwd_kernel<T, 96, 96, 2, VEC>, g, 96, st, a); break;
      case 128: rc = launch_overlapped(norm_bwd_kernel<T, 128, 128, 2, VEC>, g, 128, st, a); break;
      case 160: rc = launch_overlapped(norm_bwd_kernel<T, 160, 160, 2, VEC>, g, 160, st, a); break;
      case 256: rc = launch_overlapped(norm_bwd_kernel<T, 256, 256, 2, VEC>, g, 256, st, a); break;
      default: rc = launch_overlapped(norm_bwd_kernel<T, 512, 512, 2, VEC>, g, 512, st, a);
    }
  }
  return rc ? rc : launch_overlapped(norm_bwd_sum_kernel, (unsigned)blocks_of(a.d, 32), 1024, st, a.partial, rows, (int64_t)a.d, dw);
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
  if (d > kMostFeatures) return B2_ERR_VARIANT;
  const NormArgs a{(int)d, t, X, R, w, H, Q, S, ldx, ldr, ldh, ldq, lds, rstd, eps};
  const bool vec = columns_aligned(X, ldx, es, 16) && (!R || columns_aligned(R, ldr, es, 16)) && (!H || columns_aligned(H, ldh, es, 16)) &&
                   columns_aligned(Q, ldq, 1, 8) && columns_aligned(w, 0, es, 16);
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  if (type == B2_TYPE_BF16) return vec ? norm_launch<__nv_bfloat16, true>(a, st) : norm_launch<__nv_bfloat16, false>(a, st);
  return vec ? norm_launch<float, true>(a, st) : norm_launch<float, false>(a, st);
}

extern "C" size_t b2_rmsnorm_backward_workspace_bytes(int64_t d, int64_t t) {
  if (d <= 0 || t <= 0) return 0;
  const int64_t a = b2::bwd_rows(d, t, 2), b = b2::bwd_rows(d, t, 4);
  return b2::round_up((size_t)(a > b ? a : b) * (size_t)d * sizeof(float), 256);
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
  if (d > kMostFeatures) return B2_ERR_VARIANT;
  const NormBwdArgs a{(int)d, t, DY, H, w, DH, DX, lddy, ldh, lddh, lddx, rstd, static_cast<float*>(workspace)};
  const bool vec = columns_aligned(DY, lddy, es, 16) && columns_aligned(H, ldh, es, 16) && (!DH || columns_aligned(DH, lddh, es, 16)) &&
                   columns_aligned(DX, lddx, es, 16) && columns_aligned(w, 0, es, 16);
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  if (type == B2_TYPE_BF16) return vec ? norm_bwd_launch<__nv_bfloat16, true>(a, dw, st) : norm_bwd_launch<__nv_bfloat16, false>(a, dw, st);
  return vec ? norm_bwd_launch<float, true>(a, dw, st) : norm_bwd_launch<float, false>(a, dw, st);
}
