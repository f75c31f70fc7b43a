// Product of two block-scaled e4m3 matrices on the 5th-generation tensor cores.
//
//   C_ij = alpha * sum_b sA(i, b) sB(j, b) * ( sum_{p in block b} a_ip b_pj ) + beta * C_ij,   blocks of 128 along p
//
// The inner sums are exact products accumulated in fp32 in tensor memory; a stage of the shared-memory ring holds
// exactly one block (128 bytes of e4m3), so that the factor of a stage is a number per row times a number per column.
//
// This file has the entry points, of products alone and of those with an epilogue (f8_act.cuh); f8_small.cuh has the kernel for small products, one CTA to a tile; large ones go to
// pairs of CTAs (f8_mx.cu, f8_fs.cu).
//
// Roles of a CTA: warp 0 streams both operands with TMA (128-byte swizzle) into the ring, warp 1 issues tcgen05.mma, the other
// warps bring the scales and read the sums.  With e8m0 scales the tensor core applies them and the sums stay in tensor memory for
// as many blocks as chunk_blocks allows; otherwise every block's sums are read (two buffers in turn) and added, times the scales, to fp32
// accumulators.  A second buffer for the chunks' sums would spare the pause of 0.3 us at each (1408 x 1408 x 8192 fp32 27.0 us, 25.5 in one chunk).
//
// The matrix whose index is contiguous in C (A, index i) is the MMA's column operand (tiles 128 x 128 or 128 x 64): results leave in whole
// lines.  For few columns (decoding: n <= 64) A gives the 128 rows and the tile is as narrow as n.  The k range may be split
// over a cluster, whose CTAs add their shares through distributed shared memory.
//
// What bounds it: latencies.  1024^3 takes 5.9 us, of which the first operands take 2 and the results 1; adding shares of 128 x 128
// tiles takes 2 us (distributed shared memory delivers 14 bytes a clock), which is why narrow tiles come before splits.  Decoding
// (8192 x 8 x 8192) takes 14.5 us (calls from Python 15.0) for 64 MB of weights, 4.6 TB/s; the weights alone would take 10.3.
#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>

#include "f8_small.cuh"

namespace b2 {

extern template int f8_choose<float, true>(const F8ArgsOf<F8ActOut>&, const F8Operand&, const F8Operand&, int64_t, cudaStream_t);
extern template int f8_choose<float, false>(const F8ArgsOf<F8ActOut>&, const F8Operand&, const F8Operand&, int64_t, cudaStream_t);
extern template int f8_choose<__nv_bfloat16, true>(const F8ArgsOf<F8ActOut>&, const F8Operand&, const F8Operand&, int64_t, cudaStream_t);
extern template int f8_choose<__nv_bfloat16, false>(const F8ArgsOf<F8ActOut>&, const F8Operand&, const F8Operand&, int64_t, cudaStream_t);

namespace {

// ---- operands whose columns are not 16-byte aligned are copied into columns that are --------------------
// Both operands' in one launch: CTAs (., y) copy operand y.
__global__ void __launch_bounds__(256) f8_repitch_kernel(const F8Copy first, const F8Copy second, const FastDiv per_first, const FastDiv per_second) {
  grid_started();
  grid_ready();
  const F8Copy& p = blockIdx.y ? second : first;
  const FastDiv per = blockIdx.y ? per_second : per_first;
  const uint8_t* src = static_cast<const uint8_t*>(p.src);
  uint8_t* dst = static_cast<uint8_t*>(p.dst);
  const int64_t ld = p.ld, rows = p.rows, cols = p.cols, ldd = p.ldd;
  const int64_t total = (int64_t)per.d * cols;
  for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t c = total <= 0x7fffffffLL ? (int64_t)div_by((uint32_t)i, per) : i / per.d, r = (i - c * per.d) * 16, n = rows - r;
    const uint8_t* s = src + c * ld + r;
    uint32_t w[4] = {0, 0, 0, 0};
    if ((r > 0 || c > 0) && (n >= 20 || (c + 1 < cols && ld >= 32))) {  // up to 3 bytes before and 19 after lie within the matrix
      const uint32_t* a = reinterpret_cast<const uint32_t*>(reinterpret_cast<uintptr_t>(s) & ~(uintptr_t)3);
      const int shift = (int)(reinterpret_cast<uintptr_t>(s) & 3) * 8;
      uint32_t v[5];
#pragma unroll
      for (int j = 0; j < 5; ++j) v[j] = a[j];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        w[j] = __funnelshift_r(v[j], v[j + 1], shift);
        const int64_t left = n - 4 * j;
        if (left < 4) w[j] = left > 0 ? w[j] & (0xffffffffu >> (32 - 8 * (int)left)) : 0u;
      }
    } else {
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (j < n) w[j >> 2] |= (uint32_t)s[j] << (8 * (j & 3));
    }
    *reinterpret_cast<uint4*>(dst + c * ldd + r) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

template <typename TC>
__global__ void __launch_bounds__(256) f8_scale_c_kernel(int64_t m, int64_t n, float beta, TC* C, int64_t ldc) {
  grid_started();
  grid_ready();
  for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < m * n; i += (int64_t)gridDim.x * 256) {
    TC* c = C + i % m + i / m * ldc;
    f8_store1(c, beta == 0.0f ? 0.0f : beta * f8_load1(c));
  }
}

unsigned grid_for(int64_t threads) {
  const int64_t b = blocks_of(threads, 256), cap = (int64_t)sm_count_cached() * 16;
  return (unsigned)(b < 1 ? 1 : b < cap ? b : cap);
}

// SMs that clusters of 2^log CTAs, one to an SM, can hold at once: a cluster stays within one group of SMs, and the groups are no multiples
// of eight, nor alike on every GPU.
int f8_cluster_slots(int log) {
  static std::atomic<int> known[64][4];
  const int sms = sm_count_cached();
  int dev = -1;
  if (log == 0 || cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return sms;
  int slots = known[dev][log].load(std::memory_order_acquire);
  if (slots) return slots;
  auto kfn = f8_gemm_kernel<128, float, true, true, F8Out>;
  using Cfg = F8Cfg<128, true>;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(1, 1u << log), cfg.blockDim = Cfg::NT, cfg.dynamicSmemBytes = Cfg::SMEM;
  cudaLaunchAttribute at = {};
  at.id = cudaLaunchAttributeClusterDimension, at.val.clusterDim = {1, 1u << log, 1};
  cfg.attrs = &at, cfg.numAttrs = 1;
  int clusters = 0;
  if (cudaFuncSetAttribute(kfn, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Cfg::SMEM) != cudaSuccess ||
      cudaOccupancyMaxActiveClusters(&clusters, kfn, &cfg) != cudaSuccess || clusters < 1) {
    (void)cudaGetLastError();
    return sms * 3 / 4;
  }
  slots = clusters << log;
  known[dev][log].store(slots, std::memory_order_release);
  return slots;
}

bool f8_is_n(char c) { return c == 'N' || c == 'n'; }
bool f8_is_t(char c) { return c == 'T' || c == 't' || c == 'C' || c == 'c'; }

// Copies of operands that TMA cannot read.
struct F8Pack {
  bool a, b;
  int64_t lda, ldb;
  size_t off_b, total;
};
F8Pack f8_pack_plan(bool an, bool bn, int64_t m, int64_t n, int64_t k, const void* A, int64_t lda, const void* B, int64_t ldb) {
  F8Pack p{};
  p.a = !columns_aligned(A, lda, 1, 16), p.b = !columns_aligned(B, ldb, 1, 16);
  const int64_t ra = an ? m : k, ca = an ? k : m, rb = bn ? k : n, cb = bn ? n : k;
  p.lda = (int64_t)round_up((size_t)ra, 16), p.ldb = (int64_t)round_up((size_t)rb, 16);
  p.off_b = p.a ? round_up((size_t)p.lda * ca, 256) : 0;
  p.total = p.off_b + (p.b ? round_up((size_t)p.ldb * cb, 256) : 0);
  return p;
}

}  // namespace

// What the product takes, in clocks: turns of CTAs over the SMs, and adding the shares, half as long again for every doubling.  Without a
// split there is one CTA to an SM, which walks over its tiles (counted as if `resident` of them shared it, 50304 x 64 over 4096 with e8m0 scales was
// split: 45.6 us, 42.6 without).  CTAs of a cluster are not persistent: each further turn begins anew, 3000 clocks to its first product, and joins at its end.
// Measured with clusters that do not fit at once: weight gradient of 512 x 512 over 4096 tokens 20.1 us with 16 clusters of eight, 13.8 with four.
F8Split f8_split_for(int64_t tiles, int stages, double stage, double join, int resident) {
  F8Split best{1, 0.0};
  for (int s = 1, log = 0; s <= kMaxSplit && (s == 1 || stages / s >= 2); s *= 2, ++log) {
    const int r = s == 1 ? 1 : resident;
    const double turns = (double)blocks_of(tiles * s, (int64_t)f8_cluster_slots(log) * r), work = (double)r * (double)blocks_of(stages, s) * stage;
    const double clocks = s == 1 ? turns * work : turns * (work + join * (0.7 + 0.3 * log)) + (turns - 1.0) * 3000.0;
    if (s == 1 || clocks < best.clocks) best = {s, clocks};
  }
  return best;
}

int f8_repitch(const F8Copy* copies, int count, cudaStream_t st) {
  const F8Copy &a = copies[0], &b = copies[count - 1];
  const int64_t most = a.ldd / 16 * a.cols > b.ldd / 16 * b.cols ? a.ldd / 16 * a.cols : b.ldd / 16 * b.cols;
  return launch_overlapped(f8_repitch_kernel, dim3(grid_for(most), (unsigned)count), 256, st, a, b, fast_div((uint32_t)(a.ldd / 16)), fast_div((uint32_t)(b.ldd / 16)));
}
int f8_scale_c(int64_t m, int64_t n, float beta, void* C, int64_t ldc, int type_c, cudaStream_t st) {
  if (beta == 1.0f) return B2_OK;
  if (type_c == B2_TYPE_BF16) return launch_overlapped(f8_scale_c_kernel<__nv_bfloat16>, grid_for(m * n), 256, st, m, n, beta, static_cast<__nv_bfloat16*>(C), ldc);
  return launch_overlapped(f8_scale_c_kernel<float>, grid_for(m * n), 256, st, m, n, beta, static_cast<float*>(C), ldc);
}

}  // namespace b2

namespace b2 {
namespace {

// What the entry points' first eighteen arguments are.
struct F8Product {
  char transa, transb;
  int64_t m, n, k;
  float alpha;
  const void* A;
  int64_t lda;
  const void* SA;
  int64_t ldsa;
  int block_a, scale_type_a;
  const void* B;
  int64_t ldb;
  const void* SB;
  int64_t ldsb;
  int block_b, scale_type_b;

  bool an() const { return f8_is_n(transa); }
  bool bn() const { return f8_is_n(transb); }
  bool nonempty() const { return m > 0 && n > 0; }
  bool reads() const { return nonempty() && k > 0 && alpha != 0.0f; }
  bool mx() const { return scale_type_a == B2_SCALE_E8M0 && scale_type_b == B2_SCALE_E8M0; }
};
inline int64_t at_least_one(int64_t v) { return v > 1 ? v : 1; }

int f8_check(const F8Product& p) {
  const bool an = p.an(), bn = p.bn(), reads = p.reads();
  if (!an && !f8_is_t(p.transa)) return -1;
  if (!bn && !f8_is_t(p.transb)) return -2;
  if (p.m < 0) return -3;
  if (p.n < 0) return -4;
  if (p.k < 0) return -5;
  if (reads && !p.A) return -7;
  if (p.lda < at_least_one(an ? p.m : p.k)) return -8;
  if (reads && !p.SA) return -9;
  if (p.block_a != 1 && p.block_a != kF8Block) return -11;
  if (p.ldsa < at_least_one(an ? blocks_of(p.m, p.block_a) : blocks_of(p.k, kF8Block))) return -10;
  if (p.scale_type_a != B2_SCALE_E8M0 && p.scale_type_a != B2_SCALE_F32) return -12;
  if (reads && !p.B) return -13;
  if (p.ldb < at_least_one(bn ? p.k : p.n)) return -14;
  if (reads && !p.SB) return -15;
  if (p.block_b != 1 && p.block_b != kF8Block) return -17;
  if (p.ldsb < at_least_one(bn ? blocks_of(p.k, kF8Block) : blocks_of(p.n, p.block_b))) return -16;
  if (p.scale_type_b != B2_SCALE_E8M0 && p.scale_type_b != B2_SCALE_F32) return -18;
  return B2_OK;
}

// The product of checked operands with m, n, k > 0, copied first where TMA cannot read them.
template <typename OUT>
int f8_run(const F8Product& p, const OUT& out, int type_c, void* workspace, size_t workspace_bytes, cudaStream_t st) {
  const bool an = p.an(), bn = p.bn();
  const int64_t m = p.m, n = p.n, k = p.k;
  const void *A = p.A, *B = p.B;
  int64_t lda = p.lda, ldb = p.ldb;
  constexpr int64_t kMost = 0x7fffffffLL - 512;
  if (m > kMost || n > kMost || k > kMost) return B2_ERR_VARIANT;
  const F8Pack pk = f8_pack_plan(an, bn, m, n, k, A, lda, B, ldb);
  if (pk.total && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0 || workspace_bytes < pk.total)) return B2_ERR_WORKSPACE;
  F8Copy copies[2];
  int count = 0;
  if (pk.a) {
    copies[count++] = {A, lda, an ? m : k, an ? k : m, workspace, pk.lda};
    A = workspace, lda = pk.lda;
  }
  if (pk.b) {
    void* to = static_cast<char*>(workspace) + pk.off_b;
    copies[count++] = {B, ldb, bn ? k : n, bn ? n : k, to, pk.ldb};
    B = to, ldb = pk.ldb;
  }
  if (count) {
    const int rc = f8_repitch(copies, count, st);
    if (rc) return rc;
  }
  F8ArgsOf<OUT> a = {};
  a.out = out;
  a.kb = (int)blocks_of(k, kF8Block);
  a.chunk = type_c == B2_TYPE_F32 ? chunk_blocks<float>() : f8_whole_blocks(out) ? kChunkOfQ : chunk_blocks<__nv_bfloat16>();
  a.status = status_pointer();
  if (!a.status) return B2_ERR_LAUNCH;
  auto scale = [](const void* s, bool blocks_contiguous, int64_t ld, int block, int type) {
    return F8Scale{s, blocks_contiguous ? ld : 1, blocks_contiguous ? 1 : ld, block == 1 ? 0 : 7, type == B2_SCALE_F32,
                   type == B2_SCALE_E8M0 && blocks_contiguous && columns_aligned(s, ld, 1, 4)};
  };
  const F8Operand oa{A, m, lda, an, scale(p.SA, !an, p.ldsa, p.block_a, p.scale_type_a)};
  const F8Operand ob{B, n, ldb, !bn, scale(p.SB, bn, p.ldsb, p.block_b, p.scale_type_b)};
  if (type_c == B2_TYPE_BF16) return p.mx() ? f8_choose<__nv_bfloat16, true>(a, oa, ob, k, st) : f8_choose<__nv_bfloat16, false>(a, oa, ob, k, st);
  return p.mx() ? f8_choose<float, true>(a, oa, ob, k, st) : f8_choose<float, false>(a, oa, ob, k, st);
}

// A product without terms: a warp to a block of 128 features of a token.
template <typename TC>
__global__ void __launch_bounds__(256) act_of_nothing_kernel(const F8ActOut p, int64_t blocks) {
  grid_started();
  grid_ready();
  const int lane = threadIdx.x & 31;
  for (int64_t w = blockIdx.x * (int64_t)8 + (threadIdx.x >> 5); w < blocks * p.cols; w += (int64_t)gridDim.x * 8) {
    const int64_t token = w / blocks, block0 = (w - token * blocks) * kF8Block;
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    act_finish4<TC>(p, token, p.cols, block0 + lane, 32, p.rows, v);
    if (p.Q) act_quantise4(p, token, p.cols, block0, lane, 32, p.rows, v);
  }
}

}  // namespace
}  // namespace b2

extern "C" size_t b2_gemm_f8_workspace_bytes(char transa, char transb, int64_t m, int64_t n, int64_t k, const void* A,
                                             int64_t lda, const void* B, int64_t ldb) {
  using namespace b2;
  if ((!f8_is_n(transa) && !f8_is_t(transa)) || (!f8_is_n(transb) && !f8_is_t(transb)) || m <= 0 || n <= 0 || k <= 0) return 0;
  return f8_pack_plan(f8_is_n(transa), f8_is_n(transb), m, n, k, A, lda, B, ldb).total;
}

extern "C" int b2_gemm_f8(char transa, char transb, int64_t m, int64_t n, int64_t k, float alpha, const void* A, int64_t lda,
                          const void* SA, int64_t ldsa, int block_a, int scale_type_a, const void* B, int64_t ldb,
                          const void* SB, int64_t ldsb, int block_b, int scale_type_b, float beta, void* C, int64_t ldc,
                          int type_c, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  using namespace b2;
  const F8Product p{transa, transb, m, n, k, alpha, A, lda, SA, ldsa, block_a, scale_type_a, B, ldb, SB, ldsb, block_b, scale_type_b};
  if (const int rc = f8_check(p)) return rc;
  if (p.nonempty() && !C) return -20;
  if (ldc < at_least_one(m)) return -21;
  if (type_c != B2_TYPE_F32 && type_c != B2_TYPE_BF16) return -22;
  if (!p.nonempty()) return B2_OK;
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  if (!p.reads()) return f8_scale_c(m, n, beta, C, ldc, type_c, st);
  F8Out out = {};
  out.alpha = alpha, out.beta = beta, out.C = C, out.ldc = ldc;
  out.vec = columns_aligned(C, ldc, type_c == B2_TYPE_BF16 ? 2 : 4, 16);
  return f8_run(p, out, type_c, workspace, workspace_bytes, st);
}

extern "C" int b2_gemm_f8_act(char transa, char transb, int64_t m, int64_t n, int64_t k, float alpha, const void* A, int64_t lda,
                              const void* SA, int64_t ldsa, int block_a, int scale_type_a, const void* B, int64_t ldb,
                              const void* SB, int64_t ldsb, int block_b, int scale_type_b, int act, const float* bias, void* Z, int64_t ldz,
                              const void* R, int64_t ldr, void* C, int64_t ldc, int type, void* Q, int64_t ldq, void* S, int64_t lds,
                              void* workspace, size_t workspace_bytes, void* cuda_stream) {
  using namespace b2;
  const F8Product p{transa, transb, m, n, k, alpha, A, lda, SA, ldsa, block_a, scale_type_a, B, ldb, SB, ldsb, block_b, scale_type_b};
  if (const int rc = f8_check(p)) return rc;
  const bool gradient = (act & B2_ACT_GRADIENT) != 0, nonempty = p.nonempty();
  act &= ~B2_ACT_GRADIENT;
  const int64_t least = at_least_one(m);
  if (!act_known(act)) return -19;
  if (gradient && bias) return -20;
  if (nonempty && gradient && act != B2_ACT_NONE && !Z) return -21;
  if (Z && ldz < least) return -22;
  if (R && ldr < least) return -24;
  if (nonempty && !C && !Q) return -25;
  if (C && ldc < least) return -26;
  if (type != B2_TYPE_F32 && type != B2_TYPE_BF16) return -27;
  if (Q && ldq < least) return -29;
  if (nonempty && Q && !S) return -30;
  if (Q && lds < at_least_one(blocks_of(m, kF8Block))) return -31;
  if (!nonempty) return B2_OK;
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  const int es = type == B2_TYPE_BF16 ? 2 : 4;
  auto vec = [es](const void* M, int64_t ld) { return M && columns_aligned(M, ld, es, 16); };
  F8ActOut out = {};
  out.alpha = alpha, out.act = act, out.gradient = gradient && act != B2_ACT_NONE, out.bias = bias;
  if (gradient) out.Zin = act != B2_ACT_NONE ? Z : nullptr;
  else out.Z = Z;
  out.C = C, out.R = R, out.ldz = ldz, out.ldr = ldr, out.ldc = ldc;
  out.vz = vec(Z, ldz), out.vr = vec(R, ldr), out.vc = vec(C, ldc), out.vb = (reinterpret_cast<uintptr_t>(bias) & 15) == 0;
  out.Q = static_cast<uint8_t*>(Q), out.S = static_cast<uint8_t*>(S), out.ldq = ldq, out.lds = lds, out.vq = Q && columns_aligned(Q, ldq, 1, 16);
  if (p.reads()) return f8_run(p, out, type, workspace, workspace_bytes, st);
  out.alpha = 0.0f, out.rows = m, out.cols = n;
  const int64_t blocks = blocks_of(m, kF8Block);
  if (type == B2_TYPE_BF16) return launch_overlapped(act_of_nothing_kernel<__nv_bfloat16>, grid_for(32 * blocks * n), 256, st, out, blocks);
  return launch_overlapped(act_of_nothing_kernel<float>, grid_for(32 * blocks * n), 256, st, out, blocks);
}
