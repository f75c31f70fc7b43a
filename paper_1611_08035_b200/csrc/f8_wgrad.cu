// The weight gradient from an activation kept in 8 bits, on the 5th-generation tensor cores.
//
//   C_ij = alpha * sum_p ( q_ip * s(i/128, p) ) * y_jp + beta * C_ij        p: tokens
//
// The scale belongs to a token, which is what the sum runs over, so it cannot leave the sum as it does in
// b2_gemm_f8.  It is a power of two, though, so q*s IS a bf16 number, and the product is a bf16 one on exact operands:
// 8-bit numbers are fetched, and turned into bf16 on their way to the tensor core.
//
// Roles of a CTA: warp 0 streams 64 tokens at a time of both operands with TMA, warp 1 issues tcgen05.mma, four warps
// turn the 8-bit tile into the bf16 tile the multiply reads (128-byte swizzle), eight warps add the sums of kChunk
// tokens to fp32 accumulators in registers (two tensor-memory buffers in turn) and write C.
#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>

#include "b2gemm.h"
#include "entry.h"
#include "f8.cuh"
#include "f8_out.cuh"
#include "tcgen05.cuh"

namespace b2 {
namespace {

constexpr int kRows = 128, kTok = 64;
constexpr uint32_t kRaw = kRows * kTok, kAct = kRows * kTok * 2;  // bytes of the 8-bit and the bf16 tile of a stage
// Stages whose products are summed in tensor memory before the sum moves to registers.  The tensor core's additions
// truncate: with all 8192 tokens of a 4096 x 4096 gradient summed there the relative error of an fp32 result is 4.4e-6 and
// one-sided (mean -3.5e-6); with 16 stages, 1024 tokens, it is 3.5e-7, below an fp32 matrix product's, at the same speed.
constexpr int kChunk = 16;

struct WgArgs {
  F8Out out;
  int64_t k;
  int kb, splits;  // stages of 64 tokens, CTAs that share a tile's
  int tiles_r, tiles_c, group;
  const uint8_t* S;
  int64_t lds;
  int* status;
};

template <int TBN>
struct WgCfg {
  static constexpr int EW = 8, CW = 4;
  static constexpr int COLS = TBN / 2;
  static constexpr int NT = 512;  // four warpgroups: roles, converters, two that accumulate
  static constexpr uint32_t STAGE = kRaw + kAct + TBN * kTok * 2;
  static constexpr int STAGES = TBN == 256 ? 4 : 5;
  static constexpr uint32_t RING = STAGE * STAGES;
  static constexpr size_t SMEM = 1024 + RING + 512;
  static_assert(kRows * TBN * 4 <= RING, "the split's shares pass through the ring");
};

__device__ __forceinline__ void umma_bf16(uint32_t tmem_d, uint64_t desc_a, uint64_t desc_b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(tmem_d), "l"(desc_a), "l"(desc_b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// fp32 accumulator, both operands bf16 with their own index contiguous
__host__ __device__ constexpr uint32_t umma_idesc_bf16_mn(int m, int n) {
  return (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// Two e4m3 numbers (the upper bytes of the halves of x) times 2^(byte-127) as bf16.  With the four exponent and three
// mantissa bits moved to the top of bf16's, the number reads as its value times 2^(7-127), subnormal e4m3
// numbers as subnormal bf16 ones; f1 * f2 = 2^120 * scale puts the exponent right, exactly.
__device__ __forceinline__ uint32_t e4m3x2_to_bf16x2(uint32_t x, uint32_t f1, uint32_t f2) {
  const uint32_t r = (x & 0x80008000u) | ((x >> 4) & 0x07f007f0u);
  return mul_bf16x2(mul_bf16x2(r, f1), f2);
}

template <int TBN, typename TC>
__global__ void __launch_bounds__(WgCfg<TBN>::NT, 1)
    wgrad_kernel(const WgArgs p, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_y) {
  using Cfg = WgCfg<TBN>;
  constexpr int EW = Cfg::EW, CW = Cfg::CW, COLS = Cfg::COLS, STAGES = Cfg::STAGES;
  extern __shared__ unsigned char wg_smem_raw[];
  const uint32_t raw = smem_u32(wg_smem_raw);
  unsigned char* ring = wg_smem_raw + (((raw + 1023u) & ~1023u) - raw);
  uint64_t* full = reinterpret_cast<uint64_t*>(ring + Cfg::RING);
  uint64_t* conv = full + STAGES;
  uint64_t* empty = conv + STAGES;
  uint64_t* tfull = empty + STAGES;
  uint64_t* tempty = tfull + 2;
  uint64_t* drained = tempty + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drained + 1);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&conv[s], CW);
      mbar_init(&empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&tfull[b], 1);
      mbar_init(&tempty[b], EW);
    }
    mbar_init(drained, 1);
    mbar_fence_init();
  }
  if (warp == 1) tmem_alloc(tmem_slot, 2 * TBN);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  const int tiles = p.tiles_r * p.tiles_c, share = blockIdx.y;
  const int kb0 = (int)((int64_t)p.kb * share / p.splits), kb1 = (int)((int64_t)p.kb * (share + 1) / p.splits);
  bool ok = true;

  if (warp < 4) {
    // registers: 4 x 128 at launch; 64 + 96 + 2 x 176 = 512 after the moves
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    if (warp == 0 && lane == 0) {
      int it = 0;
      for (int tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x) {
        int tr, tc;
        tile_coords(tile, p.tiles_r, p.tiles_c, p.group, tr, tc);
        for (int kb = kb0; kb < kb1; ++kb, ++it) {
          const int s = it % STAGES, r = it / STAGES;
          if (r > 0 && !mbar_wait_bounded(&empty[s], (uint32_t)((r - 1) & 1))) {
            ok = false;
            break;
          }
          unsigned char* st = ring + (size_t)s * Cfg::STAGE;
          mbar_arrive_expect_tx(&full[s], Cfg::STAGE - kAct);
          tma_load_2d(st + kAct, &map_q, tr * kRows, kb * kTok, &full[s]);
#pragma unroll
          for (int j = 0; j < TBN / 64; ++j)
            tma_load_2d(st + kAct + kRaw + j * 8192, &map_y, tc * TBN + j * 64, kb * kTok, &full[s]);
        }
      }
      if (!ok) {
        atomicExch(p.status, (int)B2_ERR_TIMEOUT);
        for (int s = 0; s < STAGES; ++s)
          if (it > s) (void)mbar_wait_bounded(&full[s], (uint32_t)(((it - 1 - s) / STAGES) & 1), kDrainLimitNs);
      }
    } else if (warp == 1 && lane == 0) {
      constexpr uint32_t idesc = umma_idesc_bf16_mn(kRows, TBN);
      int it = 0, ch = 0;
      for (int tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x) {
        for (int kb = kb0; kb < kb1; ++kb, ++it) {
          const int s = it % STAGES, in = (kb - kb0) % kChunk, b = ch & 1;
          const uint32_t phase = (uint32_t)((it / STAGES) & 1);
          if ((in == 0 && ch >= 2 && !mbar_wait_bounded(&tempty[b], (uint32_t)(((ch >> 1) - 1) & 1))) ||
              !mbar_wait_bounded(&full[s], phase) || !mbar_wait_bounded(&conv[s], phase)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t a0 = smem_u32(ring + (size_t)s * Cfg::STAGE), b0 = a0 + kAct + kRaw;
#pragma unroll
          for (int j = 0; j < kTok / 16; ++j)  // 16 tokens an instruction: two groups of eight 128-byte rows
            umma_bf16(tmem + b * TBN, umma_desc_mn_major_sw128(a0 + j * 2048, 8192), umma_desc_mn_major_sw128(b0 + j * 2048, 8192),
                      idesc, (in | j) != 0 ? 1u : 0u);
          umma_commit(&empty[s]);
          if (in == kChunk - 1 || kb == kb1 - 1) {
            umma_commit(&tfull[b]);
            ++ch;
          }
        }
      }
      if (!ok) {
        atomicExch(p.status, (int)B2_ERR_TIMEOUT);
        umma_commit(drained);
        (void)mbar_wait_bounded(drained, 0, kDrainLimitNs);
      }
    }
  } else if (warp < 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 96;");
    const int cw = warp - 4, f = lane & 15, th = lane >> 4;  // eight features of every other token
    int it = 0;
    for (int tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x) {
      int tr, tc;
      tile_coords(tile, p.tiles_r, p.tiles_c, p.group, tr, tc);
      auto scale_of = [&](int kb) -> uint32_t {  // lanes 0-15: the warp's tokens of stage kb
        const int64_t tok = (int64_t)kb * kTok + cw * 16 + f;
        return tok < p.k ? p.S[tok * p.lds + tr] : 127u;
      };
      uint32_t next = kb0 < kb1 ? scale_of(kb0) : 127u;
      for (int kb = kb0; kb < kb1; ++kb, ++it) {
        const int s = it % STAGES;
        const uint32_t mine = next;
        if (kb + 1 < kb1) next = scale_of(kb + 1);
        if (!__all_sync(0xffffffffu, mbar_wait_bounded(&full[s], (uint32_t)((it / STAGES) & 1)) ? 1 : 0)) {
          ok = false;
          break;
        }
        unsigned char* act = ring + (size_t)s * Cfg::STAGE;
        const unsigned char* src = act + kAct;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int t = cw * 16 + 2 * i + th;
          const uint32_t byte = __shfl_sync(0xffffffffu, mine, 2 * i + th);
          // 2^120 * 2^(byte-127) = 2^e1 * 2^e2 with both factors in range; a NaN scale makes everything NaN
          const int e = (int)byte - 7, e1 = min(e, 120), e2 = e - e1;
          const uint32_t h1 = byte == kScaleNan ? 0x7fc0u : (uint32_t)(e1 + 127) << 7, h2 = byte == kScaleNan ? 0x7fc0u : (uint32_t)(e2 + 127) << 7;
          const uint32_t f1 = h1 * 0x10001u, f2 = h2 * 0x10001u;
          const uint2 w = *reinterpret_cast<const uint2*>(src + t * 128 + f * 8);
          uint4 o;
          o.x = e4m3x2_to_bf16x2(__byte_perm(w.x, 0, 0x1404), f1, f2);
          o.y = e4m3x2_to_bf16x2(__byte_perm(w.x, 0, 0x3424), f1, f2);
          o.z = e4m3x2_to_bf16x2(__byte_perm(w.y, 0, 0x1404), f1, f2);
          o.w = e4m3x2_to_bf16x2(__byte_perm(w.y, 0, 0x3424), f1, f2);
          // the pattern of e4m3's NaN is 480 to the arithmetic above
          if ((((w.x & 0x7f7f7f7fu) + 0x01010101u) | ((w.y & 0x7f7f7f7fu) + 0x01010101u)) & 0x80808080u) {
            uint32_t* po = reinterpret_cast<uint32_t*>(&o);
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if ((((j < 4 ? w.x : w.y) >> (8 * (j & 3))) & 0x7fu) == 0x7fu) po[j >> 1] |= 0x7fc0u << (16 * (j & 1));
          }
          *reinterpret_cast<uint4*>(act + (f >> 3) * 8192 + t * 128 + (((f & 7) ^ (t & 7)) << 4)) = o;
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the tensor core reads through the async proxy
        __syncwarp();
        if (lane == 0) mbar_arrive(&conv[s]);
      }
    }
    if (!ok && lane == 0) atomicExch(p.status, (int)B2_ERR_TIMEOUT);
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 176;");
    const int quad = warp & 3, half = (warp - 8) >> 2;
    const uint32_t taddr = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(half * COLS);
    float acc[COLS];
    int ch = 0;
    for (int tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x) {
      int tr, tc;
      tile_coords(tile, p.tiles_r, p.tiles_c, p.group, tr, tc);
#pragma unroll
      for (int j = 0; j < COLS; ++j) acc[j] = 0.0f;
      for (int kb = kb0; kb < kb1; kb += kChunk, ++ch) {
        const int b = ch & 1;
        if (!__all_sync(0xffffffffu, mbar_wait_bounded(&tfull[b], (uint32_t)((ch >> 1) & 1)) ? 1 : 0)) {
          ok = false;
          break;
        }
        tc_fence_after();
#pragma unroll
        for (int c0 = 0; c0 < COLS; c0 += 16) {
          uint32_t v[16];
          tmem_ld16_issue(taddr + (uint32_t)(b * TBN + c0), v);
          tmem_ld_wait16(v);
          if (c0 + 16 >= COLS) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&tempty[b]);
          }
#pragma unroll
          for (int j = 0; j < 16; ++j) acc[c0 + j] += __uint_as_float(v[j]);
        }
      }
      if (!ok) {
        if (lane == 0) atomicExch(p.status, (int)B2_ERR_TIMEOUT);
      } else if (p.splits == 1) {
        f8_emit<TC, false, COLS>(p.out, (int64_t)tr * kRows + quad * 32 + lane, (int64_t)tc * TBN + half * COLS, acc);
      } else {
        float* mine = reinterpret_cast<float*>(ring) + (size_t)half * COLS * kRows + quad * 32 + lane;
#pragma unroll
        for (int j = 0; j < COLS; ++j) mine[(size_t)j * kRows] = acc[j];
      }
    }
  }
  __syncwarp();
  if (p.splits > 1) {
    int tr, tc;
    tile_coords(blockIdx.x, p.tiles_r, p.tiles_c, p.group, tr, tc);
    f8_split_join<TC, false, TBN, EW>(p.out, ring, p.splits, share, warp >= 8 && ok ? warp - 8 : -1, warp & 3,
                                      (int64_t)tr * kRows, (int64_t)tc * TBN);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) tmem_dealloc(tmem, 2 * TBN);
}

bool wg_map(CUtensorMap* map, CUtensorMapDataType type, int elem, const void* base, int64_t inner, int64_t outer, int64_t ld,
            int box_inner, CUtensorMapSwizzle swizzle) {
  EncodeFn enc = tensor_map_encode_fn();
  if (!enc) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)outer};
  const cuuint64_t strides[1] = {(cuuint64_t)ld * elem};
  const cuuint32_t box[2] = {(cuuint32_t)box_inner, (cuuint32_t)kTok};
  const cuuint32_t estr[2] = {1, 1};
  return enc(map, type, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int TBN, typename TC>
int wg_launch(WgArgs a, int64_t m, int64_t n, int64_t k, const void* Q, int64_t ldq, const void* Y, int64_t ldy, int splits,
              cudaStream_t st) {
  using Cfg = WgCfg<TBN>;
  static std::atomic<bool> configured[64];
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return B2_ERR_LAUNCH;
  auto kfn = wgrad_kernel<TBN, TC>;
  if (!configured[dev].load(std::memory_order_acquire)) {
    if (cudaFuncSetAttribute(kfn, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Cfg::SMEM) != cudaSuccess) return B2_ERR_LAUNCH;
    configured[dev].store(true, std::memory_order_release);
  }
  CUtensorMap mq, my;
  if (!wg_map(&mq, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, Q, m, k, ldq, kRows, CU_TENSOR_MAP_SWIZZLE_NONE) ||
      !wg_map(&my, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, Y, n, k, ldy, 64, CU_TENSOR_MAP_SWIZZLE_128B))
    return B2_ERR_LAUNCH;
  const int64_t tr = blocks_of(m, kRows), tc = blocks_of(n, TBN);
  if (tr * tc > 0x7fffffffLL) return B2_ERR_VARIANT;
  a.tiles_r = (int)tr, a.tiles_c = (int)tc, a.splits = splits, a.group = 8;
  const int tiles = a.tiles_r * a.tiles_c, sms = sm_count_cached();
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = splits > 1 ? dim3((unsigned)tiles, (unsigned)splits) : dim3((unsigned)(tiles < sms ? tiles : sms));
  cfg.blockDim = dim3(Cfg::NT);
  cfg.dynamicSmemBytes = Cfg::SMEM;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim = {1, (unsigned)splits, 1};
  cfg.attrs = at, cfg.numAttrs = splits > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kfn, a, mq, my) == cudaSuccess ? B2_OK : B2_ERR_LAUNCH;
}

template <typename TC>
int wg_choose(const WgArgs& a, int64_t m, int64_t n, int64_t k, const void* Q, int64_t ldq, const void* Y, int64_t ldy, cudaStream_t st) {
  const int sms = sm_count_cached();
  if (blocks_of(m, kRows) * blocks_of(n, 256) >= sms) return wg_launch<256, TC>(a, m, n, k, Q, ldq, Y, ldy, 1, st);
  const int64_t tiles = blocks_of(m, kRows) * blocks_of(n, 128);
  int s = 1;
  while (s < 8 && tiles * s * 2 <= sms && a.kb / (s * 2) >= 2) s *= 2;
  return wg_launch<128, TC>(a, m, n, k, Q, ldq, Y, ldy, s, st);
}

struct WgPack {
  bool q, y;
  int64_t ldq, ldy;
  size_t off_y, total;
};
WgPack wg_pack_plan(int64_t m, int64_t n, int64_t k, const void* Q, int64_t ldq, const void* Y, int64_t ldy) {
  WgPack p{};
  p.q = !columns_aligned(Q, ldq, 1, 16), p.y = !columns_aligned(Y, ldy, 2, 16);
  p.ldq = (int64_t)round_up((size_t)m, 16), p.ldy = (int64_t)round_up((size_t)n, 8);
  p.off_y = p.q ? round_up((size_t)p.ldq * k, 256) : 0;
  p.total = p.off_y + (p.y ? round_up((size_t)p.ldy * 2 * k, 256) : 0);
  return p;
}

}  // namespace
}  // namespace b2

extern "C" size_t b2_wgrad_f8_workspace_bytes(int64_t m, int64_t n, int64_t k, const void* Q, int64_t ldq, const void* Y, int64_t ldy) {
  if (m <= 0 || n <= 0 || k <= 0) return 0;
  return b2::wg_pack_plan(m, n, k, Q, ldq, Y, ldy).total;
}

extern "C" int b2_wgrad_f8(int64_t m, int64_t n, int64_t k, float alpha, const void* Q, int64_t ldq, const void* S, int64_t lds,
                           const void* Y, int64_t ldy, float beta, void* C, int64_t ldc, int type_c, void* workspace,
                           size_t workspace_bytes, void* cuda_stream) {
  using namespace b2;
  if (m < 0) return -1;
  if (n < 0) return -2;
  if (k < 0) return -3;
  const bool nonempty = m > 0 && n > 0, reads = nonempty && k > 0 && alpha != 0.0f;
  auto least = [](int64_t v) { return v > 1 ? v : 1; };
  if (reads && !Q) return -5;
  if (ldq < least(m)) return -6;
  if (reads && !S) return -7;
  if (lds < least(blocks_of(m, kF8Block))) return -8;
  if (reads && !Y) return -9;
  if (ldy < least(n)) return -10;
  if (nonempty && !C) return -12;
  if (ldc < least(m)) return -13;
  if (type_c != B2_TYPE_F32 && type_c != B2_TYPE_BF16) return -14;
  if (!nonempty) return B2_OK;
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  if (!reads) return f8_scale_c(m, n, beta, C, ldc, type_c, st);
  constexpr int64_t kMost = 0x7fffffffLL - 512;
  if (m > kMost || n > kMost || k > kMost) return B2_ERR_VARIANT;
  const WgPack pk = wg_pack_plan(m, n, k, Q, ldq, Y, ldy);
  if (pk.total && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0 || workspace_bytes < pk.total)) return B2_ERR_WORKSPACE;
  if (pk.q) {
    const int rc = f8_repitch(Q, ldq, m, k, workspace, pk.ldq, st);
    if (rc) return rc;
    Q = workspace, ldq = pk.ldq;
  }
  if (pk.y) {
    void* to = static_cast<char*>(workspace) + pk.off_y;
    const int rc = f8_repitch(Y, ldy * 2, n * 2, k, to, pk.ldy * 2, st);
    if (rc) return rc;
    Y = to, ldy = pk.ldy;
  }
  WgArgs a = {};
  a.out.rows = m, a.out.cols = n, a.out.alpha = alpha, a.out.beta = beta, a.out.C = C, a.out.ldc = ldc;
  a.k = k, a.kb = (int)blocks_of(k, kTok);
  a.S = static_cast<const uint8_t*>(S), a.lds = lds;
  a.status = status_pointer();
  if (!a.status) return B2_ERR_LAUNCH;
  return type_c == B2_TYPE_BF16 ? wg_choose<__nv_bfloat16>(a, m, n, k, Q, ldq, Y, ldy, st) : wg_choose<float>(a, m, n, k, Q, ldq, Y, ldy, st);
}
