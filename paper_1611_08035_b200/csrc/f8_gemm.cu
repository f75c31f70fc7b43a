// Product of two block-scaled e4m3 matrices on the 5th-generation tensor cores.
//
//   C_ij = alpha * sum_b sA(i, b) sB(j, b) * ( sum_{p in block b} a_ip b_pj ) + beta * C_ij,   blocks of 128 along p
//
// The inner sums are exact products accumulated in fp32 in tensor memory; a stage of the shared-memory ring holds
// exactly one block (128 bytes of e4m3), so that the factor of a stage is a number per row times a number per column.
//
// This file has the entry points and the kernel for small products, one CTA to a tile; large ones go to pairs of CTAs (f8_mx.cu, f8_fs.cu).
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

#include "f8_gemm.cuh"

namespace b2 {
namespace {

// MX: both scales are e8m0 and the tensor core applies them (f8_mx.cu describes how): the sums of a chunk stay in tensor
// memory, behind them the scales of sixteen blocks.  Otherwise every block's sums are scaled and added in registers.
template <int TBN, bool MX>
struct F8Cfg {
  static constexpr int EW = TBN >= 128 ? 8 : 4;             // warps that read the sums
  static constexpr int COLS = TBN / (EW / 4);               // accumulators of a thread
  static constexpr int NT = 64 + 32 * EW;
  static constexpr uint32_t STAGE = kRowStage + TBN * kF8Block;
  static constexpr int STAGES = TBN == 128 ? 6 : TBN == 64 ? 4 : 5;
  // CTAs that an SM holds.  The one with 64 columns and scales in registers takes 177 of them a thread; kept to the 168 that two would leave it is
  // slower where one is enough (8192 x 64 x 8192 20.6 us, 19.8).  That the split's rule counted two all the same cost 50304 x 64 over 4096 71.7 us, now 49.3.
  static constexpr int RESIDENT = TBN < 64 || (TBN == 64 && MX) ? 2 : 1;
  static constexpr uint32_t RING = STAGE * STAGES;
  static constexpr int SLOTS = 4, SF_COLS = 8;              // scale ring in tensor memory: 4 columns for 128 rows, 4 for 128 columns
  static constexpr uint32_t TMEM = MX ? (TBN <= 32 ? 64 : TBN == 64 ? 128 : 256) : (TBN == 16 ? 32 : 2 * TBN);
  static_assert(!MX || TBN + SLOTS * SF_COLS <= (int)TMEM, "sums and scales");
  static constexpr int SCRATCH = kEmitBytes > COLS * 4 ? kEmitBytes : COLS * 4;  // of a warp: staged rows of C, or a block's column scales
  static constexpr size_t SMEM = 1024 + RING + 512 + EW * SCRATCH;
  static_assert(share_bytes(TBN) <= RING, "the split's shares pass through the ring");
  static_assert(RESIDENT * (SMEM + 1024) <= 228 * 1024 && RESIDENT * TMEM <= 512, "shared and tensor memory of an SM");
};

__device__ __forceinline__ void umma_f8(uint32_t tmem_d, uint64_t desc_a, uint64_t desc_b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(tmem_d), "l"(desc_a), "l"(desc_b), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void umma_mx1(uint32_t tmem_d, uint64_t desc_a, uint64_t desc_b, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                         uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
      ::"r"(tmem_d), "l"(desc_a), "l"(desc_b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
      : "memory");
}

template <int TBN, typename TC, bool COLS_CONTIG, bool MX>
__global__ void __launch_bounds__(F8Cfg<TBN, MX>::NT, F8Cfg<TBN, MX>::RESIDENT)
    f8_gemm_kernel(const F8Args p, const __grid_constant__ CUtensorMap map_r, const __grid_constant__ CUtensorMap map_c) {
  using Cfg = F8Cfg<TBN, MX>;
  constexpr int EW = Cfg::EW, COLS = Cfg::COLS, STAGES = Cfg::STAGES, CHUNK = chunk_blocks<TC>();
  extern __shared__ unsigned char f8_smem_raw[];
  const uint32_t raw = smem_u32(f8_smem_raw);
  unsigned char* ring = f8_smem_raw + (((raw + 1023u) & ~1023u) - raw);
  uint64_t* full = reinterpret_cast<uint64_t*>(ring + Cfg::RING);
  uint64_t* empty = full + STAGES;
  uint64_t* tfull = empty + STAGES;
  uint64_t* tempty = tfull + 2;
  uint64_t* sf_full = tempty + 2;
  uint64_t* sf_empty = sf_full + Cfg::SLOTS;
  uint64_t* drained = sf_empty + Cfg::SLOTS;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drained + 1);
  unsigned char* scratch = ring + Cfg::RING + 512;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    tma_prefetch_map(&map_r);
    tma_prefetch_map(&map_c);
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&tfull[b], 1);
      mbar_init(&tempty[b], EW);
    }
    for (int s = 0; s < Cfg::SLOTS; ++s) {
      mbar_init(&sf_full[s], 4);
      mbar_init(&sf_empty[s], 1);
    }
    mbar_init(drained, 1);
    mbar_fence_init();
  }
  if (warp == 1) tmem_alloc(tmem_slot, Cfg::TMEM);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  grid_ready();

  // split: the cluster's CTAs (blockIdx.y) share one tile; otherwise the grid walks over the tiles
  const int tiles = p.tiles_r * p.tiles_c, share = blockIdx.y;
  const int kb0 = (int)((int64_t)p.kb * share / p.splits), kb1 = (int)((int64_t)p.kb * (share + 1) / p.splits);
  bool ok = true;
  float acc[COLS];

  if (warp == 0) {
    if (lane == 0) {
      RingPos<STAGES> pos;
      int filled = 0;
      for (int tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x) {
        int tr, tc;
        tile_coords(tile, p.tiles_r, p.tiles_c, p.group, tr, tc);
        for (int kb = kb0; kb < kb1; ++kb, pos.next()) {
          const int s = pos.s;
          if (filled < STAGES) {
            ++filled;
          } else if (!mbar_wait_bounded(&empty[s], pos.phase ^ 1u)) {
            ok = false;
            break;
          }
          unsigned char* st = ring + (size_t)s * Cfg::STAGE;
          mbar_arrive_expect_tx(&full[s], Cfg::STAGE);
          tma_load_2d(st, &map_r, p.r_mn ? tr * kRows : kb * kF8Block, p.r_mn ? kb * kF8Block : tr * kRows, &full[s]);
          tma_load_2d(st + kRowStage, &map_c, p.c_mn ? tc * TBN : kb * kF8Block, p.c_mn ? kb * kF8Block : tc * TBN, &full[s]);
        }
      }
      if (!ok) {  // nothing of this CTA's copies may still be in flight when it leaves: the latest fill of every slot
        atomicExch(p.status, (int)B2_ERR_TIMEOUT);
        for (int i = 0; i < filled; ++i, pos.next()) (void)mbar_wait_bounded(&full[pos.s], pos.phase ^ 1u, kDrainLimitNs);
      }
    }
  } else if (warp == 1) {
    const uint32_t a0 = smem_u32(ring), b0 = a0 + kRowStage;
    const uint64_t da0 = p.r_mn ? umma_desc_mn_major_sw128(a0, kRowStage) : umma_desc_k_major_sw128(a0);
    const uint64_t db0 = !p.c_mn ? umma_desc_k_major_sw128(b0) : TBN == 64 ? umma_desc_mn_major_sw64(b0) : umma_desc_mn_major_sw128(b0, kRowStage);
    const uint32_t step_a = p.r_mn ? 4096 : 32, step_b = p.c_mn ? 32 * TBN : 32;  // bytes between instructions of a block
    const uint32_t idesc = MX ? umma_idesc_mx(kRows, TBN, p.r_mn, p.c_mn, 0) : umma_idesc_f8(kRows, TBN, p.r_mn, p.c_mn);
    RingPos<STAGES> pos;
    RingPos<Cfg::SLOTS> slot;
    int ch = 0;  // sums handed over so far: buffer and round (MX: one buffer)
    for (int tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x) {
      for (int kb = kb0; kb < kb1; ++kb, pos.next()) {
        const int s = pos.s, b = MX ? 0 : ch & 1, byte = kb & 3;
        const bool first = !MX || kb == kb0 || kb % CHUNK == 0, end = !MX || kb == kb1 - 1 || kb % CHUNK == CHUNK - 1;
        const uint32_t behind = MX ? 1 : 2, round = (uint32_t)(MX ? ch : ch >> 1);
        if ((first && ch >= (int)behind && !mbar_wait_warp(&tempty[b], (round - 1) & 1)) ||
            (MX && (byte == 0 || kb == kb0) && !mbar_wait_warp(&sf_full[slot.s], slot.phase)) ||
            !mbar_wait_warp(&full[s], pos.phase)) {
          ok = false;
          break;
        }
        tc_fence_after();
        const uint64_t da = umma_desc_advance(da0, (uint32_t)s * Cfg::STAGE), db = umma_desc_advance(db0, (uint32_t)s * Cfg::STAGE);
        const bool group_end = MX && (byte == 3 || end);
        if (elect_one()) {
          if constexpr (MX) {
            const uint32_t sfa = tmem + TBN + slot.s * Cfg::SF_COLS, id = idesc | ((uint32_t)byte << 4) | ((uint32_t)byte << 29);
#pragma unroll
            for (int j = 0; j < 4; ++j)  // 32 of the summed index an instruction
              umma_mx1(tmem, umma_desc_advance(da, j * step_a), umma_desc_advance(db, j * step_b), id, sfa, sfa + 4, (!first || j != 0) ? 1u : 0u);
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              umma_f8(tmem + b * TBN, umma_desc_advance(da, j * step_a), umma_desc_advance(db, j * step_b), idesc, j != 0 ? 1u : 0u);
          }
          umma_commit(&empty[s]);
          if (group_end) umma_commit(&sf_empty[slot.s]);
          if (end) umma_commit(&tfull[b]);
        }
        __syncwarp();
        if (group_end) slot.next();
        if (end) ++ch;
      }
    }
    if (!ok) {  // multiply-adds in flight write tensor memory: let them end before it is freed
      if (elect_one()) {
        atomicExch(p.status, (int)B2_ERR_TIMEOUT);
        umma_commit(drained);
      }
      (void)mbar_wait_warp(drained, 0, kDrainLimitNs);
    }
  } else {
    const int ew = warp - 2, quad = warp & 3, half = ew >> 2;  // tensor-memory lanes go by the warp's number modulo 4
    const uint32_t taddr = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(half * COLS);
    constexpr int SPL = (COLS + 31) / 32;
    RingPos<Cfg::SLOTS> slot;
    int ch = 0, groups = 0;
    for (int tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x) {
      int tr, tc;
      tile_coords(tile, p.tiles_r, p.tiles_c, p.group, tr, tc);
      const int64_t row = (int64_t)tr * kRows + quad * 32 + lane, col0 = (int64_t)tc * TBN + half * COLS;
      if constexpr (MX) {
        const int64_t r0 = (int64_t)tr * kRows + lane, c0 = (int64_t)tc * TBN + lane;
        constexpr int CW = TBN >= 32 ? TBN / 32 : 1;
        uint32_t next[4 + CW];
        auto fetch = [&](int kb) {
          scale_words<4>(p.sr, r0, p.out.rows, kb, p.kb, next);
          scale_words<CW>(p.sc, c0, p.out.cols, kb, p.kb, next + 4);
        };
        auto bring = [&](int kb) {  // the scales of four blocks to tensor memory
          uint32_t w[8] = {};
#pragma unroll
          for (int i = 0; i < 4 + CW; ++i) w[i] = next[i];
          if (kb + 4 < kb1) fetch(kb + 4);
          if (groups < Cfg::SLOTS) {
            ++groups;
          } else if (!mbar_wait_warp(&sf_empty[slot.s], slot.phase ^ 1u)) {
            return ok = false;
          }
          tc_fence_after();
          const uint32_t sf = tmem + ((uint32_t)(quad * 32) << 16) + TBN + slot.s * Cfg::SF_COLS;
          tmem_st4(sf, w[0], w[1], w[2], w[3]);
          tmem_st4(sf + 4, w[4], w[5], w[6], w[7]);
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&sf_full[slot.s]);
          slot.next();
          return true;
        };
        auto sums = [&](auto take) {  // of one chunk, once its last product is there
          if (!mbar_wait_warp(&tfull[0], (uint32_t)(ch & 1), kWaitLimitNs + (uint64_t)p.kb * 8192ull)) return ok = false;
          ++ch;
          tc_fence_after();
#pragma unroll
          for (int j0 = 0; j0 < COLS; j0 += 16) {
            uint32_t v[16];
            tmem_ld16_issue(taddr + (uint32_t)j0, v);
            tmem_ld_wait16(v);
#pragma unroll
            for (int j = 0; j < 16; ++j) take(acc[j0 + j], __uint_as_float(v[j]));
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&tempty[0]);
          return true;
        };
        // Four warps (half 0), one for each quarter of the lanes, bring the scales; all read the sums.
        const bool brings = half == 0;
        if (brings) fetch(kb0 & ~3);
        if (kb0 / CHUNK == (kb1 - 1) / CHUNK) {
          for (int kb = kb0 & ~3; brings && kb < kb1; kb += 4)
            if (!bring(kb)) break;
          if (ok) sums([](float& s, float v) { s = v; });
        } else {
#pragma unroll
          for (int j = 0; j < COLS; ++j) acc[j] = 0.0f;
          // The slot for the scales of block kb is the one of 4 SLOTS blocks ago.  If those began a chunk, their products wait for the sums
          // of the chunk before to be read, by these warps among others: that comes first.
          int left = (kb1 - 1) / CHUNK - kb0 / CHUNK + 1;
          for (int kb = brings ? kb0 & ~3 : kb1; left > 0; kb += 4) {
            const int behind = kb - 4 * Cfg::SLOTS;
            if (kb >= kb1 || (behind > kb0 && behind % CHUNK == 0)) {
              if (!sums([](float& s, float v) { s += v; })) break;
              --left;
            }
            if (kb < kb1 && !bring(kb)) break;
          }
        }
      } else {
        float* scw = reinterpret_cast<float*>(scratch + ew * Cfg::SCRATCH);
        const int64_t srow = row < p.out.rows ? row : p.out.rows - 1;
#pragma unroll
        for (int j = 0; j < COLS; ++j) acc[j] = 0.0f;
        float fr = 0.0f, fc[SPL];
        auto fetch = [&](int kb) {
          fr = f8_scale_at(p.sr, srow, kb);
#pragma unroll
          for (int i = 0; i < SPL; ++i) {
            int64_t c = col0 + i * 32 + (lane % COLS);
            fc[i] = f8_scale_at(p.sc, c < p.out.cols ? c : p.out.cols - 1, kb);
          }
        };
        if (kb0 < kb1) fetch(kb0);
        for (int kb = kb0; kb < kb1; ++kb, ++ch) {
          const int b = ch & 1;
          const float f = fr;
          __syncwarp();
#pragma unroll
          for (int i = 0; i < SPL; ++i)
            if (COLS >= 32 || lane < COLS) scw[i * 32 + lane] = fc[i];
          __syncwarp();
          if (kb + 1 < kb1) fetch(kb + 1);
          if (!mbar_wait_warp(&tfull[b], (uint32_t)((ch >> 1) & 1))) {
            ok = false;
            break;
          }
          tc_fence_after();
          constexpr int W = COLS >= 32 ? 32 : 16;
#pragma unroll
          for (int c0 = 0; c0 < COLS; c0 += W) {
            uint32_t v[32];
            if constexpr (W == 32) {
              tmem_ld32_issue(taddr + (uint32_t)(b * TBN + c0), v);
              tmem_ld_wait32(v);
            } else {
              uint32_t(&v16)[16] = *reinterpret_cast<uint32_t(*)[16]>(v);
              tmem_ld16_issue(taddr + (uint32_t)(b * TBN + c0), v16);
              tmem_ld_wait16(v16);
            }
            if (c0 + W >= COLS) {
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(&tempty[b]);
            }
#pragma unroll
            for (int j = 0; j < W; ++j) acc[c0 + j] += __uint_as_float(v[j]) * (f * scw[c0 + j]);
          }
        }
        __syncwarp();
      }
      if (tile + (int)gridDim.x >= tiles) grid_started();
      if (!ok) {
        if (lane == 0) atomicExch(p.status, (int)B2_ERR_TIMEOUT);
      } else if (p.splits > 1) {
        // this CTA's share of the tile; the ring is idle once the last block's sums have been read
        f8_put_share<COLS_CONTIG, TBN, COLS>(ring, quad * 32 + lane, half * COLS, acc);
      } else if constexpr (COLS_CONTIG) {
        f8_emit_staged<TC, COLS>(p.out, row - lane, col0, acc, scratch + ew * Cfg::SCRATCH);
      } else {
        f8_emit_rows<TC, COLS>(p.out, row, col0, acc);
      }
    }
  }
  __syncwarp();

  if (p.splits > 1) {
    int tr, tc;
    tile_coords(blockIdx.x, p.tiles_r, p.tiles_c, p.group, tr, tc);
    f8_split_join<TC, COLS_CONTIG, TBN, EW, false>(p.out, ring, p.splits, share, warp >= 2 ? tid - 64 : -1, ok, (int64_t)tr * kRows,
                                                   (int64_t)tc * TBN);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) tmem_dealloc(tmem, Cfg::TMEM);
}

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

template <int TBN, typename TC, bool COLS_CONTIG, bool MX>
int f8_launch(F8Args a, const F8Operand& r, const F8Operand& c, int64_t k, int splits, cudaStream_t st) {
  using Cfg = F8Cfg<TBN, MX>;
  static std::atomic<bool> configured[64];
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return B2_ERR_LAUNCH;
  auto kfn = f8_gemm_kernel<TBN, TC, COLS_CONTIG, MX>;
  if (!configured[dev].load(std::memory_order_acquire)) {
    if (cudaFuncSetAttribute(kfn, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Cfg::SMEM) != cudaSuccess) return B2_ERR_LAUNCH;
    configured[dev].store(true, std::memory_order_release);
  }
  CUtensorMap mr, mc;
  if (!f8_map(&mr, r.p, r.mn ? r.n : k, r.mn ? k : r.n, r.ld, 128) ||
      !f8_map(&mc, c.p, c.mn ? c.n : k, c.mn ? k : c.n, c.ld, c.mn ? 128 : TBN, c.mn ? TBN : 128))
    return B2_ERR_LAUNCH;
  const int64_t tr = blocks_of(r.n, kRows), tc = blocks_of(c.n, TBN);
  if (tr * tc > 0x7fffffffLL) return B2_ERR_VARIANT;
  a.out.rows = r.n, a.out.cols = c.n, a.r_mn = r.mn, a.c_mn = c.mn, a.sr = r.s, a.sc = c.s;
  a.tiles_r = (int)tr, a.tiles_c = (int)tc, a.splits = splits;
  a.group = 8;
  const int tiles = a.tiles_r * a.tiles_c, sms = sm_count_cached();
  return launch_overlapped_as(kfn, splits > 1 ? dim3((unsigned)tiles, (unsigned)splits) : dim3((unsigned)(tiles < sms ? tiles : sms)), Cfg::NT, Cfg::SMEM,
                           dim3(1, (unsigned)splits), st, a, mr, mc);
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
  auto kfn = f8_gemm_kernel<128, float, true, true>;
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

// Clocks of a block of 128 and of a join: 50 bytes of operands a clock, the rate at which one SM's copies arrived when measured, and about 30
// clocks a column of the tile.
F8Split f8_product_split(int64_t tiles, int kb, int tbn, int resident) {
  return f8_split_for(tiles, kb, (kRowStage + tbn * kF8Block) / 50.0, 30.0 * tbn, resident);
}

template <typename TC, bool MX>
int f8_choose(const F8Args& a, const F8Operand& A, const F8Operand& B, int64_t k, cudaStream_t st) {
  const int sms = sm_count_cached();
  if (B.n <= 64 && !B.mn) {  // decoding: A's rows, tiles as narrow as n
    const int tbn = B.n <= 16 ? 16 : B.n <= 32 ? 32 : 64;
    const int64_t tiles = blocks_of(A.n, kRows);
    const int resident = tbn == 16 ? F8Cfg<16, MX>::RESIDENT : tbn == 32 ? F8Cfg<32, MX>::RESIDENT : F8Cfg<64, MX>::RESIDENT;
    const int s = f8_product_split(tiles, a.kb, tbn, tiles >= sms ? resident : 1).s;
    if (tbn == 16) return f8_launch<16, TC, false, MX>(a, A, B, k, s, st);
    if (tbn == 32) return f8_launch<32, TC, false, MX>(a, A, B, k, s, st);
    return f8_launch<64, TC, false, MX>(a, A, B, k, s, st);
  }
  // pairs of CTAs as soon as single ones, with tiles a quarter of the size, would take more than one turn
  if (blocks_of(B.n, 256) * blocks_of(A.n, 256) * 4 > sms) return MX ? f8_mx_launch<TC>(a, B, A, k, st) : f8_fs_launch<TC>(a, B, A, k, st);
  const F8Split wide = f8_product_split(blocks_of(B.n, kRows) * blocks_of(A.n, 128), a.kb, 128, 1);
  const F8Split narrow = f8_product_split(blocks_of(B.n, kRows) * blocks_of(A.n, 64), a.kb, 64, 1);
  // half as many columns a tile fetch more than half as much, but spare the join when they fill the SMs without a split
  if (narrow.clocks < wide.clocks) return f8_launch<64, TC, true, MX>(a, B, A, k, narrow.s, st);
  return f8_launch<128, TC, true, MX>(a, B, A, k, wide.s, st);
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
  const bool an = f8_is_n(transa), bn = f8_is_n(transb);
  if (!an && !f8_is_t(transa)) return -1;
  if (!bn && !f8_is_t(transb)) return -2;
  if (m < 0) return -3;
  if (n < 0) return -4;
  if (k < 0) return -5;
  const bool nonempty = m > 0 && n > 0, reads = nonempty && k > 0 && alpha != 0.0f;
  auto least = [](int64_t v) { return v > 1 ? v : 1; };
  if (reads && !A) return -7;
  if (lda < least(an ? m : k)) return -8;
  if (reads && !SA) return -9;
  if (block_a != 1 && block_a != kF8Block) return -11;
  if (ldsa < least(an ? blocks_of(m, block_a) : blocks_of(k, kF8Block))) return -10;
  if (scale_type_a != B2_SCALE_E8M0 && scale_type_a != B2_SCALE_F32) return -12;
  if (reads && !B) return -13;
  if (ldb < least(bn ? k : n)) return -14;
  if (reads && !SB) return -15;
  if (block_b != 1 && block_b != kF8Block) return -17;
  if (ldsb < least(bn ? blocks_of(k, kF8Block) : blocks_of(n, block_b))) return -16;
  if (scale_type_b != B2_SCALE_E8M0 && scale_type_b != B2_SCALE_F32) return -18;
  if (nonempty && !C) return -20;
  if (ldc < least(m)) return -21;
  if (type_c != B2_TYPE_F32 && type_c != B2_TYPE_BF16) return -22;
  if (!nonempty) return B2_OK;
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  if (!reads) return f8_scale_c(m, n, beta, C, ldc, type_c, st);
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
  F8Args a = {};
  a.kb = (int)blocks_of(k, kF8Block);
  a.out.alpha = alpha, a.out.beta = beta, a.out.C = C, a.out.ldc = ldc;
  a.out.vec = columns_aligned(C, ldc, type_c == B2_TYPE_BF16 ? 2 : 4, 16);
  a.status = status_pointer();
  if (!a.status) return B2_ERR_LAUNCH;
  auto scale = [](const void* s, bool blocks_contiguous, int64_t ld, int block, int type) {
    return F8Scale{s, blocks_contiguous ? ld : 1, blocks_contiguous ? 1 : ld, block == 1 ? 0 : 7, type == B2_SCALE_F32,
                   type == B2_SCALE_E8M0 && blocks_contiguous && columns_aligned(s, ld, 1, 4)};
  };
  const F8Operand oa{A, m, lda, an, scale(SA, !an, ldsa, block_a, scale_type_a)};
  const F8Operand ob{B, n, ldb, !bn, scale(SB, bn, ldsb, block_b, scale_type_b)};
  const bool mx = scale_type_a == B2_SCALE_E8M0 && scale_type_b == B2_SCALE_E8M0;
  if (type_c == B2_TYPE_BF16) return mx ? f8_choose<__nv_bfloat16, true>(a, oa, ob, k, st) : f8_choose<__nv_bfloat16, false>(a, oa, ob, k, st);
  return mx ? f8_choose<float, true>(a, oa, ob, k, st) : f8_choose<float, false>(a, oa, ob, k, st);
}
