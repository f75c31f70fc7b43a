// The block-scaled e4m3 product on pairs of CTAs when a scale is an arbitrary fp32 number: the tensor core cannot apply
// it, so every block's sums leave tensor memory for fp32 accumulators in registers.
//
// A pair owns a 256 x 256 tile of C, operands as in f8_mx.cu.  A block of 128 is 512 clocks of tensor pipe, in which a CTA's
// eight accumulating warps read 128 x 256 sums from tensor memory (two buffers in turn) and do as many multiply-adds:
// half of the fp32 pipe, and the reason why the tile's row scale and, for 128 x 128 blocks, its column scale are made one
// factor a thread.
//
// What bounds it: those eight warps.  A block takes about 1000 clocks, 415 of them reading tensor memory (shared with the next block's
// accumulation), the others barriers, scales and multiply-adds one after the other: 4096^3 in 78-88 us (1.6-1.8 PFLOP/s), 8192^3 in 531 us.
// Sixteen warps of 64 columns read no faster (103 us); reading the next block's scales early cost registers (104 us).
//
// Warps of a CTA: 0 streams the operands (TMA), 1 issues the multiply-adds (leader only), 4-7 bring the scales of four
// blocks at a time to shared memory, 8-15 scale, add and write C.
#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>

#include "f8_gemm.cuh"

namespace b2 {
namespace {

constexpr int kBN = 256;                // columns of the pair's tile
constexpr int kStages = 3;              // operand ring
constexpr int kPerStage = 2;            // blocks of a stage
constexpr uint32_t kBlockBytes = 2 * kRowStage;
constexpr uint32_t kStageBytes = kPerStage * kBlockBytes;
constexpr uint32_t kRing = kStageBytes * kStages;
constexpr int kThreads = 512, kEW = 8, kCols = kBN / 2;
constexpr int kSlots = 2, kGroup = 4;   // scale ring: slots of four blocks
constexpr int kSlotFloats = kGroup * (kRows + kBN);  // [block][128 rows, 256 columns]
constexpr size_t kSmem = 1024 + kRing + 512 + kSlots * kSlotFloats * 4 + kEW * kEmitBytes;
static_assert(kSmem <= 232448, "a CTA's shared memory");

__device__ __forceinline__ void umma_f8_pair(uint32_t tmem_d, uint64_t desc_a, uint64_t desc_b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(tmem_d), "l"(desc_a), "l"(desc_b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// (d0, d1) = (a0, a1) * (b0, b1) + (d0, d1), and the product alone
__device__ __forceinline__ void fma2(uint64_t& d, uint64_t a, uint64_t b) { asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(d) : "l"(a), "l"(b)); }
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t pair_of(uint32_t lo, uint32_t hi) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "r"(lo), "r"(hi));
  return d;
}

// Scales of index i for blocks b .. b+3 (clamped to the last).  Rows of scales lie far apart, so the four in one load where
// they are aligned.
__device__ __forceinline__ void scales_of(const F8Scale& s, int64_t i, int b, int kb, float (&v)[kGroup]) {
  const int64_t at = (i >> s.shift) * s.si + (int64_t)b * s.sb;
  if (s.f32) {
    const float* q = static_cast<const float*>(s.p) + at;
    if (s.sb == 1 && b + kGroup <= kb && (reinterpret_cast<uintptr_t>(q) & 15) == 0) {
      const float4 f = *reinterpret_cast<const float4*>(q);
      v[0] = f.x, v[1] = f.y, v[2] = f.z, v[3] = f.w;
      return;
    }
  } else {
    const uint8_t* q = static_cast<const uint8_t*>(s.p) + at;
    if (s.sb == 1 && b + kGroup <= kb && (reinterpret_cast<uintptr_t>(q) & 3) == 0) {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(q);
#pragma unroll
      for (int g = 0; g < kGroup; ++g) v[g] = e8m0_value((w >> (8 * g)) & 255u);
      return;
    }
  }
#pragma unroll
  for (int g = 0; g < kGroup; ++g) v[g] = f8_scale_at(s, i, min(b + g, kb - 1));
}

template <typename TC>
__global__ void __launch_bounds__(kThreads, 1)
    f8_fs_kernel(const F8Args p, const __grid_constant__ CUtensorMap map_r, const __grid_constant__ CUtensorMap map_c) {
  extern __shared__ unsigned char fs_smem_raw[];
  const uint32_t raw = smem_u32(fs_smem_raw);
  unsigned char* ring = fs_smem_raw + (((raw + 1023u) & ~1023u) - raw);
  uint64_t* full = reinterpret_cast<uint64_t*>(ring + kRing);
  uint64_t* empty = full + kStages;
  uint64_t* sf_full = empty + kStages;
  uint64_t* sf_empty = sf_full + kSlots;
  uint64_t* tfull = sf_empty + kSlots;
  uint64_t* tempty = tfull + 2;
  uint64_t* drained = tempty + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drained + 1);
  float* scales = reinterpret_cast<float*>(ring + kRing + 512);

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
      mbar_init(&sf_full[s], 4);
      mbar_init(&sf_empty[s], kEW);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&tfull[b], 1);
      mbar_init(&tempty[b], 2 * kEW);
    }
    mbar_init(drained, 1);
    mbar_fence_init();
  }
  if (warp == 1) tmem_alloc_pair(tmem_slot, 2 * kBN);
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();  // the other CTA's barriers exist before anything arrives on them
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  grid_ready();
  const int tiles = p.tiles_r * p.tiles_c, pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  bool ok = true;

  // registers: 4 x 128 at launch; 40 + 56 + 2 x 208 = 512 after the moves
  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
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
      const uint32_t a0 = smem_u32(ring), b0 = a0 + kRowStage;
      const uint64_t da0 = p.r_mn ? umma_desc_mn_major_sw128(a0, kRowStage) : umma_desc_k_major_sw128(a0);
      const uint64_t db0 = p.c_mn ? umma_desc_mn_major_sw128(b0, kRowStage) : umma_desc_k_major_sw128(b0);
      const uint32_t step_a = p.r_mn ? 4096 : 32, step_b = p.c_mn ? 4096 : 32;  // bytes between instructions of a block
      const uint32_t idesc = umma_idesc_f8(2 * kRows, kBN, p.r_mn, p.c_mn);
      int ch = 0;  // blocks so far: buffer and round
      bool ready = false;
      for (int tile = pair; tile < tiles && ok; tile += pairs) {
        for (int kb = 0; kb < p.kb && ok; kb += kPerStage) {
          const int s = pos.s, here = min(kPerStage, p.kb - kb);
          if (!ready && !mbar_wait_warp(&full[s], pos.phase)) {
            ok = false;
            break;
          }
          for (int h = 0; h < here; ++h, ++ch) {
            const int b = ch & 1;
            if (ch >= 2 && !mbar_wait_warp(&tempty[b], (uint32_t)(((ch >> 1) - 1) & 1))) {
              ok = false;
              break;
            }
            tc_fence_after();
            const uint64_t da = umma_desc_advance(da0, (uint32_t)s * kStageBytes + h * kBlockBytes);
            const uint64_t db = umma_desc_advance(db0, (uint32_t)s * kStageBytes + h * kBlockBytes);
            if (elect_one()) {
#pragma unroll
              for (int j = 0; j < 4; ++j)
                umma_f8_pair(tmem + b * kBN, umma_desc_advance(da, j * step_a), umma_desc_advance(db, j * step_b), idesc, j != 0 ? 1u : 0u);
              umma_commit_pair(&tfull[b]);
              if (h == here - 1) umma_commit_pair(&empty[s]);
            }
            __syncwarp();
          }
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
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    const int i = tid - 128;
    RingPos<kSlots> slot;
    int filled = 0;
    for (int tile = pair; tile < tiles && ok; tile += pairs) {
      int tr, tc;
      tile_coords(tile, p.tiles_r, p.tiles_c, p.group, tr, tc);
      const int64_t r = min((int64_t)tr * 2 * kRows + rank * kRows + i, p.out.rows - 1);
      const int64_t c0 = min((int64_t)tc * kBN + i, p.out.cols - 1), c1 = min((int64_t)tc * kBN + 128 + i, p.out.cols - 1);
      float next[kGroup][3];  // the following group's scales are fetched while this one waits for its slot
      auto fetch = [&](int kb) {
        float v[kGroup];
        scales_of(p.sr, r, kb, p.kb, v);
#pragma unroll
        for (int g = 0; g < kGroup; ++g) next[g][0] = v[g];
        scales_of(p.sc, c0, kb, p.kb, v);
#pragma unroll
        for (int g = 0; g < kGroup; ++g) next[g][1] = v[g];
        scales_of(p.sc, c1, kb, p.kb, v);
#pragma unroll
        for (int g = 0; g < kGroup; ++g) next[g][2] = v[g];
      };
      fetch(0);
      for (int kb = 0; kb < p.kb; kb += kGroup, slot.next()) {
        if (filled < kSlots) {
          ++filled;
        } else if (!mbar_wait_warp(&sf_empty[slot.s], slot.phase ^ 1u)) {
          ok = false;
          break;
        }
        float* to = scales + slot.s * kSlotFloats + i;
#pragma unroll
        for (int g = 0; g < kGroup; ++g) {
          to[g * (kRows + kBN)] = next[g][0];
          to[g * (kRows + kBN) + kRows] = next[g][1];
          to[g * (kRows + kBN) + kRows + 128] = next[g][2];
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&sf_full[slot.s]);
        if (kb + kGroup < p.kb) fetch(kb + kGroup);
      }
    }
    if (!ok && lane == 0) atomicExch(p.status, (int)B2_ERR_TIMEOUT);
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    const int quad = warp & 3, half = (warp - 8) >> 2;
    const uint32_t taddr = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(half * kCols);
    const uint32_t leader_tempty = cluster_map_shared(smem_u32(tempty), 0);
    unsigned char* stage = ring + kRing + 512 + kSlots * kSlotFloats * 4 + (warp - 8) * kEmitBytes;
    RingPos<kSlots> slot;
    uint64_t acc2[kCols / 2];
    const bool one_factor = p.sc.shift == 7;  // the columns of a half share a scale
    int ch = 0;
    for (int tile = pair; tile < tiles && ok; tile += pairs) {
      int tr, tc;
      tile_coords(tile, p.tiles_r, p.tiles_c, p.group, tr, tc);
      f8_prefetch<TC>(p.out, true, (int64_t)tr * 2 * kRows + rank * kRows + quad * 32, 32, (int64_t)tc * kBN + half * kCols, kCols);
#pragma unroll
      for (int j = 0; j < kCols / 2; ++j) acc2[j] = 0;
      for (int kb = 0; kb < p.kb; ++kb, ++ch) {
        const int b = ch & 1, g = kb % kGroup;
        if (g == 0 && !mbar_wait_warp(&sf_full[slot.s], slot.phase)) {
          ok = false;
          break;
        }
        const float* sc = scales + slot.s * kSlotFloats + g * (kRows + kBN);
        const float fr = sc[quad * 32 + lane];
        const float* fc = sc + kRows + half * kCols;
        const uint32_t f = __float_as_uint(fr * fc[0]);
        const uint64_t ff = pair_of(f, f), rr = pair_of(__float_as_uint(fr), __float_as_uint(fr));
        auto add = [&](int c, const uint32_t (&v)[32]) {
          if (one_factor) {
#pragma unroll
            for (int j = 0; j < 16; ++j) fma2(acc2[16 * c + j], pair_of(v[2 * j], v[2 * j + 1]), ff);
          } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const ulonglong2 q = *reinterpret_cast<const ulonglong2*>(fc + 32 * c + 4 * j);
              fma2(acc2[16 * c + 2 * j], pair_of(v[4 * j], v[4 * j + 1]), mul2(q.x, rr));
              fma2(acc2[16 * c + 2 * j + 1], pair_of(v[4 * j + 2], v[4 * j + 3]), mul2(q.y, rr));
            }
          }
        };
        if (!mbar_wait_warp(&tfull[b], (uint32_t)((ch >> 1) & 1))) {
          ok = false;
          break;
        }
        tc_fence_after();
        // four loads of 32 columns through two sets of registers, each on its way while an earlier one is added
        const uint32_t from = taddr + (uint32_t)(b * kBN);
        uint32_t v0[32], v1[32];
        tmem_ld32_issue(from, v0);
        tmem_ld32_issue(from + 32, v1);
        tmem_ld_wait32(v0);
        tmem_ld_wait32(v1);
        add(0, v0);
        tmem_ld32_issue(from + 64, v0);
        add(1, v1);
        tmem_ld_wait32(v0);
        tmem_ld32_issue(from + 96, v1);
        add(2, v0);
        tmem_ld_wait32(v1);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(leader_tempty + 8u * b);
        add(3, v1);
        if (g == kGroup - 1 || kb == p.kb - 1) {
          __syncwarp();
          if (lane == 0) mbar_arrive(&sf_empty[slot.s]);
          slot.next();
        }
      }
      if (tile + pairs >= tiles) grid_started();
      const int64_t row0 = (int64_t)tr * 2 * kRows + rank * kRows + quad * 32, col0 = (int64_t)tc * kBN + half * kCols;
      float acc[kCols];
#pragma unroll
      for (int j = 0; j < kCols / 2; ++j) {
        uint32_t lo, hi;
        asm("mov.b64 {%0, %1}, %2;" : "=r"(lo), "=r"(hi) : "l"(acc2[j]));
        acc[2 * j] = __uint_as_float(lo), acc[2 * j + 1] = __uint_as_float(hi);
      }
      if (!ok) {
        if (lane == 0) atomicExch(p.status, (int)B2_ERR_TIMEOUT);
      } else {
        f8_emit_staged<TC, kCols>(p.out, row0, col0, acc, stage);
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();  // the pair's instructions read both CTAs' memory: neither leaves first
  if (warp == 1) tmem_dealloc_pair(tmem, 2 * kBN);
}

}  // namespace

template <typename TC>
int f8_fs_launch(F8Args a, const F8Operand& r, const F8Operand& c, int64_t k, cudaStream_t st) {
  static std::atomic<bool> configured[64];
  return f8_pair_launch(f8_fs_kernel<TC>, configured, kThreads, kSmem, a, r, c, k, st);
}
template int f8_fs_launch<float>(F8Args, const F8Operand&, const F8Operand&, int64_t, cudaStream_t);
template int f8_fs_launch<__nv_bfloat16>(F8Args, const F8Operand&, const F8Operand&, int64_t, cudaStream_t);

}  // namespace b2
