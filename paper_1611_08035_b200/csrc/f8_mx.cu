// The block-scaled e4m3 product with power-of-two scales applied by the tensor core itself
// (tcgen05.mma kind::mxf8f6f4, one e8m0 factor per row or column and 32 elements of the summed index: the four
// instructions of a block of 128 take the same one), on pairs of CTAs.
//
// A pair owns a 256 x 256 tile of C: each CTA fetches its 128 rows of the row operand and its 128 columns of the
// column operand, so that shared memory is written and read 32 KB per block and SM where a CTA alone would need 48 for the same
// multiply-adds; the leader's tensor core instruction reads both halves.  The sums of a chunk of blocks stay in tensor
// memory (256 columns); 48 more columns hold the scales of sixteen blocks.
//
// What bounds it: power.  8192^3 takes 383 us in a burst and 440 us on and on (2.5 PFLOP/s), a block 581 clocks where the tensor pipe
// needs 512, at 1.3 GHz under the board's power limit; without the limit (4096^3, one turn of four not full) 55 us.  Steps on the
// way, 8192^3: 599 us with every warp fetching all scales, 501 with each word fetched once, 434 with two blocks a stage and a
// converged issuing warp (its own instructions, 795 clocks a block, were what the pipe waited for), 407 with results staged for whole
// lines, 383 without cluster-scope release on arrivals.
//
// With an epilogue (OUT = F8ActTiles, f8_act.cuh): 16384 x 8192 x 4096 from 404 us in a burst to 412 with C through shared memory and TMA, 434 with bias, gelu, z and an 8-bit result, 436 with bias and
// residual, 494 as the gradient of gelu with C and an 8-bit result, whose warps take longer for a tile (21,000 clocks) than the tensor core (18,600).
//
// Warps of a CTA: 0 streams the operands (TMA), 1 issues the multiply-adds (leader only), 4-7 put the scales
// into tensor memory, four blocks at a time (byte = block, lane and column = row), 8-15 write C.
#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>
#include <type_traits>

#include "f8_gemm.cuh"

namespace b2 {
namespace {

constexpr int kBN = 256;                       // columns of the pair's tile
constexpr int kStages = 3, kSlots = 4;         // operand ring, scale ring
constexpr int kPerStage = 2;                   // blocks of a stage
constexpr uint32_t kBlockBytes = 2 * kRowStage;  // a CTA's halves of both operands, a block
constexpr uint32_t kStageBytes = kPerStage * kBlockBytes;
constexpr uint32_t kRing = kStageBytes * kStages;
constexpr int kThreads = 512, kEW = 8, kCols = kBN / 2;
constexpr uint32_t kTmem = 512, kSfCols = 12;  // scales of four blocks: 128 rows in 4 columns, 256 columns in 8
constexpr uint32_t kSfBytes = 2 * kSfCols * 32 * 4;
template <typename OUT>
constexpr size_t kSmem = 1024 + kRing + 512 + kSfBytes + kEW * ActHandOver<OUT>::WARP_BYTES;
static_assert(kSmem<F8ActTiles<3, false>> <= 232448, "a CTA's shared memory");

__device__ __forceinline__ void umma_mx(uint32_t tmem_d, uint64_t desc_a, uint64_t desc_b, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                        uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
      ::"r"(tmem_d), "l"(desc_a), "l"(desc_b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
      : "memory");
}
// CHUNKS: false where all blocks fit one chunk: then the accumulators are read once and no register holds them before.
template <typename TC, bool CHUNKS, typename OUT>
__global__ void __launch_bounds__(kThreads, 1)
    f8_mx_kernel(const __grid_constant__ F8ArgsOf<OUT> p, const __grid_constant__ CUtensorMap map_r, const __grid_constant__ CUtensorMap map_c) {
  extern __shared__ unsigned char mx_smem_raw[];
  const uint32_t raw = smem_u32(mx_smem_raw);
  unsigned char* ring = mx_smem_raw + (((raw + 1023u) & ~1023u) - raw);
  uint64_t* full = reinterpret_cast<uint64_t*>(ring + kRing);
  uint64_t* empty = full + kStages;
  uint64_t* sf_full = empty + kStages;
  uint64_t* sf_empty = sf_full + kSlots;
  uint64_t* tfull = sf_empty + kSlots;
  uint64_t* tempty = tfull + 1;
  uint64_t* drained = tempty + 1;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drained + 1);
  uint32_t* sf_words = reinterpret_cast<uint32_t*>(ring + kRing + 512);  // [2][kSfCols][32]

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_rank();
  if (tid == 0) {
    tma_prefetch_map(&map_r);
    tma_prefetch_map(&map_c);
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int s = 0; s < kSlots; ++s) {
      mbar_init(&sf_full[s], 8);  // four warps of each CTA
      mbar_init(&sf_empty[s], 1);
    }
    mbar_init(tfull, 1);
    mbar_init(tempty, 2 * kEW);
    mbar_init(drained, 1);
    mbar_fence_init();
  }
  if (warp == 1) tmem_alloc_pair(tmem_slot, kTmem);
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();  // the other CTA's barriers exist before anything arrives on them
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  grid_ready();
  const int tiles = p.tiles_r * p.tiles_c, pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const int chunk = chunk_blocks_of<TC>(p);
  bool ok = true;

  if (warp < 4) {
    // registers: 4 x 128 at launch; 64 + 80 + 2 x 184 = 512 after the moves
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    if (warp == 0 && lane == 0) {
      RingPos<kStages> pos;
      int filled = 0;  // stages that have been filled at least once
      const uint32_t leader_full = cluster_map_shared(smem_u32(full), 0);
      for (int tile = pair; tile < tiles && ok; tile += pairs) {
        int tr, tc;
        tile_coords(tile, p.tiles_r, p.tiles_c, p.group, tr, tc);
        const int r0 = tr * 2 * kRows + (int)rank * kRows, c0 = tc * kBN + (int)rank * (kBN / 2);
        for (int kb = 0; kb < p.kb; kb += kPerStage, pos.next()) {
          const int s = pos.s, here = min(kPerStage, p.kb - kb);
          if (filled < kStages) {
            ++filled;
          } else if (!mbar_wait_bounded(&empty[s], pos.phase ^ 1u)) {
            ok = false;
            break;
          }
          if (rank == 0) mbar_arrive_expect_tx(&full[s], 2 * kBlockBytes * here);
          for (int h = 0; h < here; ++h) {
            unsigned char* st = ring + (size_t)s * kStageBytes + (size_t)h * kBlockBytes;
            const int k0 = (kb + h) * kF8Block;
            tma_load_2d_pair(st, &map_r, p.r_mn ? r0 : k0, p.r_mn ? k0 : r0, leader_full + 8u * s);
            tma_load_2d_pair(st + kRowStage, &map_c, p.c_mn ? c0 : k0, p.c_mn ? k0 : c0, leader_full + 8u * s);
          }
        }
      }
      if (!ok) {
        atomicExch(p.status, (int)B2_ERR_TIMEOUT);
        if (rank == 0)  // both CTAs' copies are counted here; no CTA leaves before the barrier at the end
          for (int i = 0; i < filled; ++i, pos.next()) (void)mbar_wait_bounded(&full[pos.s], pos.phase ^ 1u, kDrainLimitNs);
      }
    } else if (warp == 1 && rank == 0) {
      RingPos<kStages> pos;
      RingPos<kSlots> slot;
      const uint32_t a0 = smem_u32(ring), b0 = a0 + kRowStage;
      const uint64_t da0 = p.r_mn ? umma_desc_mn_major_sw128(a0, kRowStage) : umma_desc_k_major_sw128(a0);
      const uint64_t db0 = p.c_mn ? umma_desc_mn_major_sw128(b0, kRowStage) : umma_desc_k_major_sw128(b0);
      const uint32_t step_a = p.r_mn ? 4096 : 32, step_b = p.c_mn ? 4096 : 32;  // bytes between instructions of a block
      const uint32_t idesc0 = umma_idesc_mx(2 * kRows, kBN, p.r_mn, p.c_mn, 0);
      // The instructions of a stage go out as fast as the tensor core takes them, one or two ahead of the one it works on; what
      // this warp does between two stages is free only as far as those cover it.  Hence two blocks to a stage, and a look
      // at the next stage's barrier, which is usually complete, right after.
      int ch = 0, in = 0;
      bool ready = false;
      for (int tile = pair; tile < tiles && ok; tile += pairs) {
        for (int kb = 0; kb < p.kb; kb += kPerStage) {
          const int s = pos.s, byte = kb & 3;
          if ((!ready && !mbar_wait_warp(&full[s], pos.phase)) || (byte == 0 && !mbar_wait_warp(&sf_full[slot.s], slot.phase)) ||
              (in == 0 && ch > 0 && !mbar_wait_warp(tempty, (uint32_t)((ch - 1) & 1)))) {
            ok = false;
            break;
          }
          tc_fence_after();
          const bool two = kb + 1 < p.kb, last = kb + 2 >= p.kb, end = last || (CHUNKS && in + kPerStage == chunk);
          const uint64_t da = umma_desc_advance(da0, (uint32_t)s * kStageBytes), db = umma_desc_advance(db0, (uint32_t)s * kStageBytes);
          const uint32_t sfa = tmem + kBN + slot.s * kSfCols, idesc = idesc0 | ((uint32_t)byte << 4) | ((uint32_t)byte << 29);
          if (elect_one()) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              umma_mx(tmem, umma_desc_advance(da, j * step_a), umma_desc_advance(db, j * step_b), idesc, sfa, sfa + 4, (in | j) != 0 ? 1u : 0u);
            if (two) {
              constexpr uint32_t next_byte = (1u << 4) | (1u << 29);  // byte is even
#pragma unroll
              for (int j = 0; j < 4; ++j)
                umma_mx(tmem, umma_desc_advance(da, kBlockBytes + j * step_a), umma_desc_advance(db, kBlockBytes + j * step_b), idesc | next_byte, sfa,
                        sfa + 4, 1u);
            }
            umma_commit_pair(&empty[s]);
            if (byte == 2 || last) umma_commit_pair(&sf_empty[slot.s]);
            if (end) umma_commit_pair(tfull);
          }
          __syncwarp();
          if (byte == 2 || last) slot.next();
          in += kPerStage;
          if (end) ++ch, in = 0;
          pos.next();
          ready = mbar_test_warp(&full[pos.s], pos.phase);
        }
      }
      if (!ok) {
        if (elect_one()) {
          atomicExch(p.status, (int)B2_ERR_TIMEOUT);
          umma_commit_pair(drained);
        }
        (void)mbar_wait_warp(drained, 0, kDrainLimitNs);
      }
    }
  } else if (warp < 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
    const int quad = warp & 3;
    const uint32_t sf = tmem + kBN + ((uint32_t)(quad * 32) << 16);
    int grp = 0;
    bool go = true;  // what the four warps agree on; ok is this warp's own
    for (int tile = pair; tile < tiles && go; tile += pairs) {
      int tr, tc;
      tile_coords(tile, p.tiles_r, p.tiles_c, p.group, tr, tc);
      const int64_t r0 = (int64_t)tr * 2 * kRows + rank * kRows + lane, c0 = (int64_t)tc * kBN + lane;
      // Tensor memory wants every word four times, once for each quarter of its lanes.  Each warp fetches a quarter of the
      // words, one group ahead, and the four swap them through shared memory: rows of scales lie far apart, so fetching is what
      // these warps spend their time on (all of them fetching all: 8192^3 514 us).
      uint32_t next[3];
      auto fetch = [&](int kb) {
        scale_words<1>(p.sr, r0 + 32 * quad, p.out.rows, kb, p.kb, next);
        scale_words<2>(p.sc, c0 + 64 * quad, p.out.cols, kb, p.kb, next + 1);
      };
      fetch(0);
      for (int kb = 0; kb < p.kb; kb += 4, ++grp) {
        const int slot = grp % kSlots, r = grp / kSlots;
        uint32_t* words = sf_words + (grp & 1) * kSfCols * 32 + lane;
        words[quad * 32] = next[0], words[(4 + 2 * quad) * 32] = next[1], words[(5 + 2 * quad) * 32] = next[2];
        go = named_barrier_all<1, 128>(ok);  // also: everyone has read the buffer of two groups ago
        if (!go) break;
        if (kb + 4 < p.kb) fetch(kb + 4);
        uint32_t w[kSfCols];
#pragma unroll
        for (int i = 0; i < (int)kSfCols; ++i) w[i] = words[i * 32];
        if (r > 0 && !mbar_wait_warp(&sf_empty[slot], (uint32_t)((r - 1) & 1))) {
          ok = false;
          continue;  // to the barrier where the others are told
        }
        tc_fence_after();
#pragma unroll
        for (int i = 0; i < 3; ++i) tmem_st4(sf + slot * kSfCols + 4 * i, w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(cluster_map_shared(smem_u32(&sf_full[slot]), 0));
      }
    }
    if (!ok && lane == 0) atomicExch(p.status, (int)B2_ERR_TIMEOUT);
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 184;");
    const int quad = warp & 3, half = (warp - 8) >> 2;
    const uint32_t taddr = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(half * kCols);
    const uint32_t leader_tempty = cluster_map_shared(smem_u32(tempty), 0);
    const uint64_t limit = kWaitLimitNs + (uint64_t)p.kb * 8192ull;  // outlasts the k loop that it waits for
    unsigned char* stage = ring + kRing + 512 + kSfBytes + (warp - 8) * ActHandOver<OUT>::WARP_BYTES;
    constexpr bool TILES = ActHandOver<OUT>::TILES;
    [[maybe_unused]] ActPieces<3> pieces{stage};
    float acc[kCols];
    int ch = 0;
    for (int tile = pair; tile < tiles && ok; tile += pairs) {
      int tr, tc;
      tile_coords(tile, p.tiles_r, p.tiles_c, p.group, tr, tc);
      if constexpr (!CHUNKS || TILES) f8_prefetch<TC>(p.out, true, (int64_t)tr * 2 * kRows + rank * kRows + quad * 32, 32, (int64_t)tc * kBN + half * kCols, kCols);
      if constexpr (TILES) act_begin_tile<TC>(p.out, (int64_t)tr * 2 * kRows + rank * kRows + quad * 32, (int64_t)tc * kBN + half * kCols, pieces);
      if constexpr (CHUNKS) {
#pragma unroll
        for (int j = 0; j < kCols; ++j) acc[j] = 0.0f;
      }
      for (int kb = 0; kb < p.kb; kb += CHUNKS ? chunk : p.kb, ++ch) {
        if (!mbar_wait_warp(tfull, (uint32_t)(ch & 1), limit)) {
          ok = false;
          break;
        }
        tc_fence_after();
        if constexpr (!CHUNKS) {
          uint32_t v[kCols / 32][32];
#pragma unroll
          for (int i = 0; i < kCols / 32; ++i) tmem_ld32_issue(taddr + 32 * i, v[i]);
#pragma unroll
          for (int i = 0; i < kCols / 32; ++i) {
            tmem_ld_wait32(v[i]);
#pragma unroll
            for (int j = 0; j < 32; ++j) acc[32 * i + j] = __uint_as_float(v[i][j]);
          }
        } else {
#pragma unroll
          for (int c0 = 0; c0 < kCols; c0 += 32) {
            uint32_t v[32];
            tmem_ld32_issue(taddr + c0, v);
            tmem_ld_wait32(v);
#pragma unroll
            for (int j = 0; j < 32; ++j) acc[c0 + j] += __uint_as_float(v[j]);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(leader_tempty);
      }
      if (tile + pairs >= tiles) grid_started();
      const int64_t row0 = (int64_t)tr * 2 * kRows + rank * kRows + quad * 32, col0 = (int64_t)tc * kBN + half * kCols;
      if (!ok) {
        if (lane == 0) atomicExch(p.status, (int)B2_ERR_TIMEOUT);
      } else if constexpr (TILES) {
        act_emit_tile<TC>(p.out, row0, col0, acc, pieces);
      } else {
        f8_emit_staged<TC, kCols>(p.out, row0, col0, acc, stage);
      }
    }
    if constexpr (TILES) pieces.drain();
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();  // the pair's instructions read both CTAs' memory: neither leaves first
  if (warp == 1) tmem_dealloc_pair(tmem, kTmem);
}

}  // namespace

template <typename TC, typename OUT>
int f8_mx_launch(F8ArgsOf<OUT> a, const F8Operand& r, const F8Operand& c, int64_t k, cudaStream_t st) {
  if constexpr (std::is_same<OUT, F8ActOut>::value) {
    F8ActTiles<3, false> tiles;
    F8ActTiles<3, true> gradient;
    if (f8_act_tiles<TC>(a.out, r.n, c.n, tiles)) return f8_mx_launch<TC>(f8_args_with(a, tiles), r, c, k, st);
    if (f8_act_tiles<TC>(a.out, r.n, c.n, gradient)) return f8_mx_launch<TC>(f8_args_with(a, gradient), r, c, k, st);
  }
  static std::atomic<bool> configured[64];
  if constexpr (sizeof(TC) == 2 && !ActHandOver<OUT>::TILES) {
    static std::atomic<bool> configured_whole[64];
    if (a.kb <= chunk_blocks_of<TC>(a)) return f8_pair_launch(f8_mx_kernel<TC, false, OUT>, configured_whole, kThreads, kSmem<OUT>, a, r, c, k, st);
  }
  return f8_pair_launch(f8_mx_kernel<TC, true, OUT>, configured, kThreads, kSmem<OUT>, a, r, c, k, st);
}
template int f8_mx_launch<float>(F8ArgsOf<F8Out>, const F8Operand&, const F8Operand&, int64_t, cudaStream_t);
template int f8_mx_launch<__nv_bfloat16>(F8ArgsOf<F8Out>, const F8Operand&, const F8Operand&, int64_t, cudaStream_t);
template int f8_mx_launch<float>(F8ArgsOf<F8ActOut>, const F8Operand&, const F8Operand&, int64_t, cudaStream_t);
template int f8_mx_launch<__nv_bfloat16>(F8ArgsOf<F8ActOut>, const F8Operand&, const F8Operand&, int64_t, cudaStream_t);

}  // namespace b2
