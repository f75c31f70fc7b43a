// The weight gradient from an activation kept in 8 bits, on the 5th-generation tensor cores.
//
//   C_ij = alpha * sum_p ( q_ip * s(i/128, p) ) * y_jp + beta * C_ij        p: tokens
//
// The scale belongs to a token, which is what the sum runs over, so it cannot leave the sum as it does in
// b2_gemm_f8.  It is a power of two, though, so q*s IS a bf16 number, and the product is a bf16 one on exact operands:
// 8-bit numbers are fetched, and turned into bf16 on their way to the tensor core.
//
// Large gradients go to pairs of CTAs (256 features by 256 columns of Y, cta_group::2), small ones to single CTAs (128 x 128)
// whose k range may be shared by a cluster.  Either way a CTA fetches and converts 128 features by 64 tokens a stage and
// fetches 128 columns of Y.
//
// Roles of a CTA: warp 0 streams 64 tokens at a time of both operands with TMA, warp 1 issues tcgen05.mma (of a pair:
// the leader's), warps 4-11 turn the 8-bit tile into the bf16 tile the multiply reads (128-byte swizzle), warps 12-19 add
// the sums of kChunk stages to fp32 accumulators in registers (two tensor-memory buffers in turn) and write C.
//
// What bounds it: the conversion's instructions.  A stage is 512 clocks of tensor pipe and takes 750, in which the SM issues 2300 of 3000
// possible instructions, three quarters of them conversion (30 for eight numbers, 5 of which look for NaNs, 3 % of the time); shared
// memory, at 128 bytes a clock, would need 640 (24 KB written by TMA, 8 read and 16 written by the conversion, 32 read by the multiply).
// 4096 x 4096 x 8192 takes 230 us in a burst (1.19 PFLOP/s) and 275 on and on; its 256 tiles are 3.5 turns of 74 pairs.
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

template <int CTAS>
struct WgCfg {
  static constexpr int TBN = CTAS * 128;  // columns of the tile
  static constexpr int EW = 8, CW = 4;    // warps that accumulate, warps that convert a stage (two groups of them in turn)
  static constexpr int COLS = TBN / 2;
  static constexpr int NT = 640;  // five warpgroups: roles, two that convert, two that accumulate
  static constexpr uint32_t YTILE = 128 * kTok * 2, STAGE = kRaw + kAct + YTILE;
  static constexpr int STAGES = 5;
  static constexpr uint32_t RING = STAGE * STAGES, TMEM = 2 * TBN;
  static constexpr size_t SMEM = 1024 + RING + 512;
  static_assert(share_bytes(128) <= RING, "the split's shares pass through the ring");
};

template <int CTAS>
__device__ __forceinline__ void umma_bf16(uint32_t tmem_d, uint64_t desc_a, uint64_t desc_b, uint32_t idesc, uint32_t accumulate) {
  if constexpr (CTAS == 2) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(tmem_d), "l"(desc_a), "l"(desc_b), "r"(idesc), "r"(accumulate)
        : "memory");
  } else {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(tmem_d), "l"(desc_a), "l"(desc_b), "r"(idesc), "r"(accumulate)
        : "memory");
  }
}
template <int CTAS>
__device__ __forceinline__ void wg_commit(uint64_t* bar) {
  if constexpr (CTAS == 2) umma_commit_pair(bar);
  else umma_commit(bar);
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
// Four e4m3 numbers b0..b3 of a word as bf16 pairs (b0, b2) and (b1, b3) times 2^-120: with the four exponent and three
// mantissa bits at the top of bf16's, subnormal numbers become subnormal ones and nothing is rounded.  Splitting the word
// into even and odd bytes saves the permutations that the order b0..b3 would take; the product's rows are in the same order, and
// are put back where they are written (kept_row).
__device__ __forceinline__ uint32_t e4m3_even(uint32_t w) { return ((w << 8) & 0x80008000u) | ((w << 4) & 0x07f007f0u); }
__device__ __forceinline__ uint32_t e4m3_odd(uint32_t w) { return (w & 0x80008000u) | ((w >> 4) & 0x07f007f0u); }

// Eight e4m3 numbers to bf16, times 2^120 * scale.
__device__ __forceinline__ uint4 e4m3x8_to_bf16(uint2 w, uint32_t f1) {
  return make_uint4(mul_bf16x2(e4m3_even(w.x), f1), mul_bf16x2(e4m3_odd(w.x), f1), mul_bf16x2(e4m3_even(w.y), f1),
                    mul_bf16x2(e4m3_odd(w.y), f1));
}
// bit 7 of a byte of the result is set where the number (or its carry's neighbour) may be e4m3's NaN, 0x7f
__device__ __forceinline__ uint32_t e4m3_nan_bits(uint2 w) {
  return (((w.x & 0x7f7f7f7fu) + 0x01010101u) | ((w.y & 0x7f7f7f7fu) + 0x01010101u)) & 0x80808080u;
}
// The arithmetic above reads a NaN as 480: put NaNs where the numbers are NaN.
__device__ __forceinline__ uint4 e4m3x8_nans(uint2 w, uint4 o) {
  auto fix = [](uint32_t word, int lo, int hi, uint32_t r) {
    if (((word >> (8 * lo)) & 0x7fu) == 0x7fu) r |= 0x7fc0u;
    if (((word >> (8 * hi)) & 0x7fu) == 0x7fu) r |= 0x7fc00000u;
    return r;
  };
  return make_uint4(fix(w.x, 0, 2, o.x), fix(w.x, 1, 3, o.y), fix(w.y, 0, 2, o.z), fix(w.y, 1, 3, o.w));
}

template <int CTAS, typename TC>
__global__ void __launch_bounds__(WgCfg<CTAS>::NT, 1)
    wgrad_kernel(const WgArgs p, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_y) {
  using Cfg = WgCfg<CTAS>;
  constexpr int EW = Cfg::EW, CW = Cfg::CW, COLS = Cfg::COLS, STAGES = Cfg::STAGES, TBN = Cfg::TBN;
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
  const uint32_t rank = CTAS == 2 ? cluster_rank() : 0;
  if (tid == 0) {
    tma_prefetch_map(&map_q);
    tma_prefetch_map(&map_y);
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(&full[s], 3);
      mbar_init(&conv[s], CTAS * CW);
      mbar_init(&empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&tfull[b], 1);
      mbar_init(&tempty[b], CTAS * EW);
    }
    mbar_init(drained, 1);
    mbar_fence_init();
  }
  if (warp == 1) {
    if (CTAS == 2) tmem_alloc_pair(tmem_slot, Cfg::TMEM);
    else tmem_alloc(tmem_slot, Cfg::TMEM);
  }
  tc_fence_before();
  __syncthreads();
  if (CTAS == 2) cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  grid_ready();

  const int tiles = p.tiles_r * p.tiles_c, share = CTAS == 2 ? 0 : blockIdx.y;
  const int first = blockIdx.x / CTAS, stride = gridDim.x / CTAS;
  const int kb0 = (int)((int64_t)p.kb * share / p.splits), kb1 = (int)((int64_t)p.kb * (share + 1) / p.splits);
  // address of a barrier of the CTA that issues the multiply-adds
  auto leader = [&](uint64_t* bar) { return CTAS == 2 ? cluster_map_shared(smem_u32(bar), 0) : smem_u32(bar); };
  auto arrive_leader = [&](uint32_t addr) {
    if (CTAS == 2) mbar_arrive_cluster(addr);
    else asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(addr) : "memory");
  };
  bool ok = true;

  // registers: 5 x 96 at launch; 40 + 2 x 64 + 2 x 152 = 472 after the moves
  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    if (warp != 1) {
      // warp 0 fetches the activation, warps 2 and 3 half of Y's columns each: one thread issuing all three boxes of a stage
      // needs about 1000 clocks for them
      RingPos<STAGES> pos;
      int filled = 0;
      const CUtensorMap* map = warp == 0 ? &map_q : &map_y;
      const uint32_t bytes = warp == 0 ? kRaw : Cfg::YTILE / 2, at = warp == 0 ? kAct : kAct + kRaw + (warp - 2) * (Cfg::YTILE / 2);
      for (int tile = first; tile < tiles && ok; tile += stride) {
        int tr, tc;
        tile_coords(tile, p.tiles_r, p.tiles_c, p.group, tr, tc);
        if (sizeof(TC) == 2 && warp == 3) f8_prefetch<TC>(p.out, false, (int64_t)tc * TBN, TBN, (int64_t)(tr * CTAS + (int)rank) * kRows, kRows);
        const int x = warp == 0 ? (tr * CTAS + (int)rank) * kRows : tc * TBN + (int)rank * 128 + (warp - 2) * 64;
        for (int kb = kb0; kb < kb1; ++kb, pos.next()) {
          const int s = pos.s;
          if (filled < STAGES) {
            ++filled;
          } else if (!mbar_wait_warp(&empty[s], pos.phase ^ 1u)) {
            ok = false;
            break;
          }
          if (elect_one()) {
            mbar_arrive_expect_tx(&full[s], bytes);
            tma_load_2d(ring + (size_t)s * Cfg::STAGE + at, map, x, kb * kTok, &full[s]);
          }
          __syncwarp();
        }
      }
      if (!ok) {
        if (lane == 0) atomicExch(p.status, (int)B2_ERR_TIMEOUT);
        for (int i = 0; i < filled; ++i, pos.next()) (void)mbar_wait_warp(&full[pos.s], pos.phase ^ 1u, kDrainLimitNs);
      }
    } else if (warp == 1 && rank == 0) {
      constexpr uint32_t idesc = umma_idesc_bf16_mn(CTAS * kRows, TBN);
      const uint32_t base = smem_u32(ring);
      const uint64_t da0 = umma_desc_mn_major_sw128(base, 8192), db0 = umma_desc_mn_major_sw128(base + kAct + kRaw, 8192);
      RingPos<STAGES> pos;
      int ch = 0, in = 0;
      for (int tile = first; tile < tiles && ok; tile += stride) {
        for (int kb = kb0; kb < kb1; ++kb) {
          const int s = pos.s, b = ch & 1;
          // a converted stage has also been fetched: whoever converted it had waited for both operands
          if (!mbar_wait_warp(&conv[s], pos.phase) ||
              (in == 0 && ch >= 2 && !mbar_wait_warp(&tempty[b], (uint32_t)(((ch >> 1) - 1) & 1)))) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint64_t da = umma_desc_advance(da0, (uint32_t)s * Cfg::STAGE), db = umma_desc_advance(db0, (uint32_t)s * Cfg::STAGE);
          const bool end = in == kChunk - 1 || kb == kb1 - 1;
          if (elect_one()) {
#pragma unroll
            for (int j = 0; j < kTok / 16; ++j)  // 16 tokens an instruction: two groups of eight 128-byte rows
              umma_bf16<CTAS>(tmem + b * TBN, umma_desc_advance(da, j * 2048), umma_desc_advance(db, j * 2048), idesc, (in | j) != 0 ? 1u : 0u);
            wg_commit<CTAS>(&empty[s]);
            if (end) wg_commit<CTAS>(&tfull[b]);
          }
          __syncwarp();
          ++in;
          if (end) ++ch, in = 0;
          pos.next();
        }
      }
      if (!ok) {
        if (elect_one()) {
          atomicExch(p.status, (int)B2_ERR_TIMEOUT);
          wg_commit<CTAS>(drained);
        }
        (void)mbar_wait_warp(drained, 0, kDrainLimitNs);
      }
    }
    if (CTAS == 1 && p.splits > 1) {
      f8_join_begin();
      f8_join_end();
    }
  } else if (warp < 12) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    // The two warpgroups convert every other stage each, a warp 16 tokens of it: what a stage costs besides the conversion (the
    // wait, the proxy fence, the arrival) then has the time of two stages to hide in.
    const int group = (warp - 4) >> 2, t0 = (warp & 3) * 16, f = lane & 15, th = lane >> 4;  // eight features of every other token
    const uint32_t dst0 = (uint32_t)((f >> 3) * 8192 + t0 * 128), src0 = kAct + t0 * 128 + f * 8;
    RingPos<STAGES> pos;
    for (int tile = first; tile < tiles && ok; tile += stride) {
      int tr, tc;
      tile_coords(tile, p.tiles_r, p.tiles_c, p.group, tr, tc);
      const int64_t blk = min((int64_t)tr * CTAS + rank, (p.out.rows - 1) / kF8Block);  // the tile may begin beyond the last feature
      // Scales of two of this group's stages at a time, one token a lane, fetched while the two before are converted.
      auto scales_of = [&](int kb) -> uint32_t {
        const int64_t tok = (int64_t)(kb + 2 * th) * kTok + t0 + f;
        return tok < p.k ? p.S[tok * p.lds + blk] : 127u;
      };
      uint32_t next = scales_of(kb0 + group), h = 0;
      bool large = false;
      for (int kb = kb0, own = 0; kb < kb1; ++kb, pos.next()) {
        if (((kb - kb0) & 1) != group) continue;
        if ((own & 1) == 0) {
          // 2^120 * 2^(byte-127) = 2^e1 * 2^e2, both factors in range; a NaN scale makes everything NaN
          const int e = (int)next - 7, e1 = min(e, 127), e2 = e - e1;
          h = next == kScaleNan ? 0x7fc07fc0u : (uint32_t)(e1 + 127) << 7 | (uint32_t)(e2 + 127) << 23;
          large = e2 > 0;
          next = scales_of(kb + 4);
        }
        const int s = pos.s;
        if (!mbar_wait_warp(&full[s], pos.phase)) {
          ok = false;
          break;
        }
        unsigned char* st = ring + (size_t)s * Cfg::STAGE;
        uint2 w[8];
        uint32_t nans = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = *reinterpret_cast<const uint2*>(st + src0 + (2 * i + th) * 128);
        const int src_lane = (own & 1) * 16 + th;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int t = 2 * i + th;
          const uint32_t hh = __shfl_sync(0xffffffffu, h, src_lane + 2 * i);
          nans |= e4m3_nan_bits(w[i]);
          *reinterpret_cast<uint4*>(st + dst0 + t * 128 + (((f ^ t) & 7) << 4)) =
              e4m3x8_to_bf16(w[i], __byte_perm(hh, 0, 0x1010));
        }
        // Rare, and therefore apart: branches among the eight conversions above would keep the compiler from overlapping them.
        if (__any_sync(0xffffffffu, large || nans != 0)) {
#pragma unroll 1
          for (int i = 0; i < 8; ++i) {
            const int t = 2 * i + th;
            const uint32_t f2 = __byte_perm(__shfl_sync(0xffffffffu, h, src_lane + 2 * i), 0, 0x3232);
            uint4* o = reinterpret_cast<uint4*>(st + dst0 + t * 128 + (((f ^ t) & 7) << 4));
            const uint4 v = make_uint4(mul_bf16x2(o->x, f2), mul_bf16x2(o->y, f2), mul_bf16x2(o->z, f2), mul_bf16x2(o->w, f2));
            *o = e4m3x8_nans(*reinterpret_cast<const uint2*>(st + src0 + t * 128), v);
          }
        }
        __syncwarp();
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the tensor core reads through the async proxy
        __syncwarp();
        if (lane == 0) arrive_leader(leader(&conv[s]));
        ++own;
      }
    }
    if (!ok && lane == 0) atomicExch(p.status, (int)B2_ERR_TIMEOUT);
    if (CTAS == 1 && p.splits > 1) {
      f8_join_begin();
      f8_join_end();
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 152;");
    const int quad = warp & 3, half = (warp - 12) >> 2;
    const uint32_t taddr = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(half * COLS);
    float acc[COLS];
    int ch = 0;
    for (int tile = first; tile < tiles && ok; tile += stride) {
      int tr, tc;
      tile_coords(tile, p.tiles_r, p.tiles_c, p.group, tr, tc);
#pragma unroll
      for (int j = 0; j < COLS; ++j) acc[j] = 0.0f;
      for (int kb = kb0; kb < kb1; kb += kChunk, ++ch) {
        const int b = ch & 1;
        if (!mbar_wait_warp(&tfull[b], (uint32_t)((ch >> 1) & 1))) {
          ok = false;
          break;
        }
        tc_fence_after();
#pragma unroll
        for (int c0 = 0; c0 < COLS; c0 += 16) {
          uint32_t v[16];
          tmem_ld16_issue(taddr + (uint32_t)(b * TBN + c0), v);
          tmem_ld_wait16(v);
#pragma unroll
          for (int j = 0; j < 16; ++j) acc[c0 + j] += __uint_as_float(v[j]);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) arrive_leader(leader(&tempty[b]));
      }
      if (tile + stride >= tiles) grid_started();
      if (!ok) {
        if (lane == 0) atomicExch(p.status, (int)B2_ERR_TIMEOUT);
      } else if (p.splits == 1) {
        f8_emit_rows<TC, COLS>(p.out, (int64_t)(tr * CTAS + (int)rank) * kRows + quad * 32 + kept_row(lane), (int64_t)tc * TBN + half * COLS, acc);
      } else {
        if constexpr (CTAS == 1) f8_put_share<false, TBN, COLS>(ring, quad * 32 + lane, half * COLS, acc);
      }
    }
    if constexpr (CTAS == 1) {
      if (p.splits > 1) {
        int tr, tc;
        tile_coords(blockIdx.x, p.tiles_r, p.tiles_c, p.group, tr, tc);
        f8_split_join<TC, false, TBN, EW, true>(p.out, ring, p.splits, share, tid - 384, ok, (int64_t)tr * kRows, (int64_t)tc * TBN);
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (CTAS == 2) cluster_sync_all();  // the pair's instructions read both CTAs' memory: neither leaves first
  if (warp == 1) {
    if (CTAS == 2) tmem_dealloc_pair(tmem, Cfg::TMEM);
    else tmem_dealloc(tmem, Cfg::TMEM);
  }
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

template <int CTAS, typename TC>
int wg_launch(WgArgs a, int64_t m, int64_t n, int64_t k, const void* Q, int64_t ldq, const void* Y, int64_t ldy, int splits,
              cudaStream_t st) {
  using Cfg = WgCfg<CTAS>;
  static std::atomic<bool> configured[64];
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return B2_ERR_LAUNCH;
  auto kfn = wgrad_kernel<CTAS, TC>;
  if (!configured[dev].load(std::memory_order_acquire)) {
    if (cudaFuncSetAttribute(kfn, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Cfg::SMEM) != cudaSuccess) return B2_ERR_LAUNCH;
    configured[dev].store(true, std::memory_order_release);
  }
  CUtensorMap mq, my;
  if (!wg_map(&mq, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, Q, m, k, ldq, kRows, CU_TENSOR_MAP_SWIZZLE_NONE) ||
      !wg_map(&my, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, Y, n, k, ldy, 64, CU_TENSOR_MAP_SWIZZLE_128B))
    return B2_ERR_LAUNCH;
  const int64_t tr = blocks_of(m, CTAS * kRows), tc = blocks_of(n, Cfg::TBN);
  if (tr * tc > 0x3fffffffLL) return B2_ERR_VARIANT;
  a.tiles_r = (int)tr, a.tiles_c = (int)tc, a.splits = splits, a.group = 8;
  const int tiles = a.tiles_r * a.tiles_c, resident = sm_count_cached() / CTAS;
  return launch_overlapped_as(kfn, splits > 1 ? dim3((unsigned)tiles, (unsigned)splits) : dim3((unsigned)((tiles < resident ? tiles : resident) * CTAS)), Cfg::NT,
                           Cfg::SMEM, dim3(CTAS, (unsigned)splits), st, a, mq, my);
}

template <typename TC>
int wg_choose(const WgArgs& a, int64_t m, int64_t n, int64_t k, const void* Q, int64_t ldq, const void* Y, int64_t ldy, cudaStream_t st) {
  const int sms = sm_count_cached();
  if (blocks_of(m, 256) * blocks_of(n, 256) * 4 > sms) return wg_launch<2, TC>(a, m, n, k, Q, ldq, Y, ldy, 1, st);
  const int64_t tiles = blocks_of(m, kRows) * blocks_of(n, 128);
  const int s = f8_split_for(tiles, a.kb, 730.0, 30.0 * 128, 1).s;  // a stage takes 0.38 us of conversion
  return wg_launch<1, TC>(a, m, n, k, Q, ldq, Y, ldy, s, st);
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
  F8Copy copies[2];
  int count = 0;
  if (pk.q) {
    copies[count++] = {Q, ldq, m, k, workspace, pk.ldq};
    Q = workspace, ldq = pk.ldq;
  }
  if (pk.y) {
    void* to = static_cast<char*>(workspace) + pk.off_y;
    copies[count++] = {Y, ldy * 2, n * 2, k, to, pk.ldy * 2};
    Y = to, ldy = pk.ldy;
  }
  if (count) {
    const int rc = f8_repitch(copies, count, st);
    if (rc) return rc;
  }
  WgArgs a = {};
  a.out.rows = m, a.out.cols = n, a.out.alpha = alpha, a.out.beta = beta, a.out.C = C, a.out.ldc = ldc;
  a.k = k, a.kb = (int)blocks_of(k, kTok);
  a.S = static_cast<const uint8_t*>(S), a.lds = lds;
  a.status = status_pointer();
  if (!a.status) return B2_ERR_LAUNCH;
  return type_c == B2_TYPE_BF16 ? wg_choose<__nv_bfloat16>(a, m, n, k, Q, ldq, Y, ldy, st) : wg_choose<float>(a, m, n, k, Q, ldq, Y, ldy, st);
}
