// Products of microscaled 4-bit operands (kernel_mx_gemm.cuh has the mathematics, layouts and orientation) on PAIRS of SMs:
// a cluster of two CTAs computes tiles of 256 output channels x 192 tokens with tcgen05.mma.cta_group::2.  Each CTA loads
// the codes of its own 128 channels and of half the tokens, the scales of its channels and of all the tokens; per
// multiply-add that is 0.61 of the bytes of a 128 x 128 tile (7 / 12 of the codes'), and bytes are what bounds long prompts.
//
// 8192 x 8192 x 8192 alone, in a captured graph: 193 to 199 us, 5.6 PFLOP/s (3.4 times the measured bf16 rate); one pass among others,
// under the power limit, 231.  What bounds it is filling shared memory: 31 KB a
// stage at the 64 bytes a cycle an SM takes in are 496 cycles, its MMAs 384, measured 590 (without the loads 430, without the
// scale copies 590).
//
// The kernel is persistent, and the epilogue of a tile runs beside the products of the next: two accumulators of 192
// columns and a place for the scales of each ring stage fill the 512 columns of tensor memory.  (The accumulators of tiles of
// 256 tokens have to overlap; the MMAs then waited some 2200 cycles from one tile to the next.)  A token tile may begin in
// the middle of a scale tile: its scales then start two columns on.
//
// Outputs whose rows are 16-byte aligned and a multiple of 16 bytes long leave through shared memory and bulk stores,
// whole rows of 128 channels; stored by the lanes a token is four pieces of 32 channels (2048 x 16384 x 1024 bf16 27.2 us, with
// 16383 channels 31.9; 8192 x 8192 x 8192 and x 8191 the same).
//
// Roles per CTA (320 threads): warp 0 lane 0 issues the loads, warp 1 owns tensor memory (lane 0 of the first CTA issues
// scale copies and MMAs for both), warps 2-9 are the epilogue: tensor-memory lanes warp % 4, one half of the columns each.
// Barriers as in kernel_igemm_pair.cuh: a stage's "full" lives in the first CTA and counts both CTAs' bytes; "empty" and
// "accumulator full" arrive in both by multicast commits; "accumulator free" lives in the first CTA.  All waits on them are bounded;
// why the cluster's own barriers and the allocation of tensor memory end is in tensor_memory.cuh.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <cstdint>
#include "kernel_igemm_pair.cuh"
#include "kernel_mx_gemm.cuh"

namespace qc {

constexpr int kMxPairThreads = 64 + 32 * 8;
constexpr int kMxPairStages = 5;
constexpr int kMxPairTokens = 192;                                       // columns of a tile
constexpr int kMxPairCols = 512;                                         // of tensor memory
constexpr uint32_t kMxPairA = 128 * kMxStageBytes, kMxPairB = kMxPairTokens / 2 * kMxStageBytes;
constexpr uint32_t kMxPairScaleB = 4 * kMxTileBytes;                     // of the 256 tokens whose scale tiles a tile touches
constexpr uint32_t kMxPairStage = kMxPairA + kMxPairB + 2 * kMxTileBytes + kMxPairScaleB;
constexpr int kMxPairScaleCol = 2 * kMxPairTokens, kMxPairScaleCols = 24;
static_assert(kMxPairScaleCol + kMxPairStages * kMxPairScaleCols <= kMxPairCols && kMxPairStage % 1024 == 0);

struct MxPairShared {
  uint64_t full[kMxPairStages];
  uint64_t empty[kMxPairStages];
  uint64_t acc_full[2];
  uint64_t acc_free[2];
  uint64_t drained;
  uint32_t tmem_base;
  volatile int abort_flag;
};
constexpr int kMxPairChunks = kMxPairTokens / 64;                         // of 32 tokens, in each half of the columns
// Staged outputs of one half of the columns: a buffer holds kBatch chunks of [32 tokens][128 channels]: a whole tile of a
// 16-bit type, or a chunk of float32 at a time in two buffers.
template <typename Y> struct MxPairOut {
  static constexpr uint32_t kChunkBytes = 32 * 128 * sizeof(Y);
  static constexpr int kBatch = sizeof(Y) == 2 ? kMxPairChunks : 1, kBuffers = sizeof(Y) == 2 ? 1 : 2;
  static constexpr uint32_t kBufferBytes = kBatch * kChunkBytes;
  static constexpr uint32_t kBytes = 2 * kBuffers * kBufferBytes;
};
template <typename Y, bool STAGED>
constexpr size_t kMxPairSmem = 1024 + kMxPairStages * kMxPairStage + (STAGED ? MxPairOut<Y>::kBytes : 0) + sizeof(MxPairShared);

namespace ptx {
__device__ __forceinline__ void mma_mxf4_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t sa_tmem,
                                              uint32_t sb_tmem, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
      ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sa_tmem), "r"(sb_tmem), "r"(accumulate)
      : "memory");
}
// Shared-memory tile -> global tensor, clipped to its extent.
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, uint32_t src, int c0, int c1) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];"
               ::"l"(reinterpret_cast<uint64_t>(map)), "r"(src), "r"(c0), "r"(c1) : "memory");
}
// All but the N most recent groups of this thread's bulk stores have read their source.
template <int N> __device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void sts_u16(uint32_t addr, uint32_t v) {
  asm volatile("st.shared.u16 [%0], %1;" ::"r"(addr), "h"(static_cast<unsigned short>(v)) : "memory");
}
__device__ __forceinline__ void sts_u32(uint32_t addr, uint32_t v) { asm volatile("st.shared.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }
__device__ __forceinline__ void st_cluster_u32(uint32_t cluster_addr, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster_addr), "r"(v) : "memory");
}
__device__ __forceinline__ void mbar_arrive_cluster_relaxed(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// Each CTA's scale tile at this shared-memory offset to its own tensor memory.
__device__ __forceinline__ void tmem_copy_scales_pair(uint32_t taddr, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
}  // namespace ptx

// Bounded wait with the hardware's suspend hint (one CTA an SM on long stages).
__device__ __forceinline__ bool mx_wait_hint(uint32_t bar, uint32_t parity, unsigned int limit, volatile int* abort_flag, int* status) {
  for (unsigned int it = 0; it < limit; ++it) {
    if (ptx::mbar_try_wait_hint(bar, parity)) return true;
    if (*abort_flag) return false;
  }
  *abort_flag = 1;
  atomicExch(status, kStatusTimeout);
  return false;
}

// Barriers of the four epilogue warps of one half of the columns; the second one also tells whether any of them failed.
__device__ __forceinline__ void mx_half_sync(int id) { asm volatile("bar.sync %0, 128;" ::"r"(id) : "memory"); }
__device__ __forceinline__ bool mx_half_vote(int id, bool failed) {
  uint32_t any;
  asm volatile(
      "{\n\t.reg .pred pin, pout;\n\t"
      "setp.ne.u32 pin, %1, 0;\n\t"
      "bar.red.or.pred pout, %2, 128, pin;\n\t"
      "selp.u32 %0, 1, 0, pout;\n\t}"
      : "=r"(any) : "r"(failed ? 1u : 0u), "r"(id) : "memory");
  return any != 0;
}

// Two values rounded to 16 bits, the first one low; negative ones to 0 with RELU (NaN stays).
template <bool RELU> __device__ __forceinline__ uint32_t mx_pack(float a, float b, __nv_bfloat16) {
  uint32_t r;
  if constexpr (RELU) asm("cvt.rn.relu.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}
template <bool RELU> __device__ __forceinline__ uint32_t mx_pack(float a, float b, __half) {
  uint32_t r;
  if constexpr (RELU) asm("cvt.rn.relu.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}
// A lane's sums of BATCH chunks, from chunk k0 on, to its channel of the staged rows.
template <typename Y, int BATCH, bool RELU>
__device__ __forceinline__ void mx_stage(uint32_t mine, const uint32_t (&acc)[kMxPairChunks][32], int k0, float b) {
#pragma unroll
  for (int k = 0; k < BATCH; ++k)
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
      const float v0 = __uint_as_float(acc[k0 + k][i]) + b, v1 = __uint_as_float(acc[k0 + k][i + 1]) + b;
      const uint32_t row = static_cast<uint32_t>(k * 32 + i) * 128 * sizeof(Y);
      if constexpr (sizeof(Y) == 2) {
        const uint32_t w = mx_pack<RELU>(v0, v1, Y());
        ptx::sts_u16(mine + row, w);
        ptx::sts_u16(mine + row + 128 * sizeof(Y), w >> 16);
      } else {
        ptx::sts_u32(mine + row, __float_as_uint(RELU && v0 < 0.0f ? 0.0f : v0));
        ptx::sts_u32(mine + row + 128 * sizeof(Y), __float_as_uint(RELU && v1 < 0.0f ? 0.0f : v1));
      }
    }
}

// Tile u of the walk: groups of eight token tiles, within a group channel tile after channel tile, so that pairs that run
// side by side share both operands in L2.
struct MxPairTile { int n0, t0; };
__device__ __forceinline__ MxPairTile mx_pair_tile(const MxGemmParams& p, int u) {
  const int per_group = 8 * p.tiles_n;
  const int g = u / per_group, in = u - g * per_group;
  const int wide = min(8, p.tiles_t - 8 * g);
  const int tn = in / wide;
  return {tn * 256, (8 * g + in - tn * wide) * kMxPairTokens};
}

template <typename Y, bool STAGED>
__global__ void __launch_bounds__(kMxPairThreads, 1)
mx_gemm_pair_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x,
                    const __grid_constant__ CUtensorMap map_ws, const __grid_constant__ CUtensorMap map_xs,
                    const __grid_constant__ CUtensorMap map_y, const MxGemmParams prm, const float* __restrict__ bias, Y* __restrict__ y,
                    int* status, unsigned int wait_limit) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint8_t* out = ring + kMxPairStages * kMxPairStage;        // STAGED: [half][buffer][chunk][32 tokens][128 channels]
  MxPairShared* sh = reinterpret_cast<MxPairShared*>(out + (STAGED ? MxPairOut<Y>::kBytes : 0));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = ptx::cluster_ctarank();
  const int pair = static_cast<int>(blockIdx.x) >> 1, pairs = static_cast<int>(gridDim.x) >> 1;
  const int total = prm.tiles_n * prm.tiles_t;
  const uint32_t ring_addr = ptx::smem_u32(ring);

  if (threadIdx.x == 0) {
    for (int s = 0; s < kMxPairStages; ++s) {
      ptx::mbar_init(ptx::smem_u32(&sh->full[s]), 1);
      ptx::mbar_init(ptx::smem_u32(&sh->empty[s]), 1);
    }
    for (int b = 0; b < 2; ++b) {
      ptx::mbar_init(ptx::smem_u32(&sh->acc_full[b]), 1);
      ptx::mbar_init(ptx::smem_u32(&sh->acc_free[b]), 2 * 8);              // epilogue warps of both CTAs
    }
    ptx::mbar_init(ptx::smem_u32(&sh->drained), 1);
    sh->abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    ptx::fence_async_smem();
    ptx::prefetch_tmap(&map_w);
    ptx::prefetch_tmap(&map_x);
    ptx::prefetch_tmap(&map_ws);
    ptx::prefetch_tmap(&map_xs);
  }
  if (warp == 1) {
    ptx::tmem_alloc_pair(ptx::smem_u32(&sh->tmem_base), kMxPairCols);
    ptx::tmem_relinquish_pair();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::cluster_sync_all();                                   // the peer's barriers exist from here on
  ptx::tc_fence_after();
  const uint32_t tmem = sh->tmem_base;
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();

  // Both issuing warps run their loops with warp-uniform values, so that addresses, coordinates and descriptors live in
  // uniform registers, where copies and MMAs take their operands from; one lane issues.
  if (warp == 0) {
    // ------------------------------------------------------------------ loads of this CTA's parts
    const bool leader = ptx::elect_one();
    bool ok = true;
    int stage = 0;
    uint32_t phase = 1;                                      // (the first pass over the ring finds every stage free)
    const int peer_row = static_cast<int>(rank) * 128;
    for (int u = pair; u < total && ok; u += pairs) {
      const MxPairTile tile = mx_pair_tile(prm, u);
      const int n0 = tile.n0 + peer_row, t0 = tile.t0 + static_cast<int>(rank) * (kMxPairTokens / 2);
      for (int kb = 0; kb < prm.k_stages; ++kb) {
        const uint32_t empty = ptx::smem_u32(&sh->empty[stage]);
        if (wait_limit == 0u || !ptx::mbar_try_wait(empty, phase)) {
          ok = mx_wait_hint(empty, phase, wait_limit, &sh->abort_flag, status);
          if (!ok) break;
        }
        const uint32_t full = ptx::smem_u32(&sh->full[stage]), full0 = ptx::map_to_cta(full, 0u);
        const uint32_t a = ring_addr + static_cast<uint32_t>(stage) * kMxPairStage;
        if (leader) {
          if (rank == 0) ptx::mbar_expect_tx(full, 2 * kMxPairStage);
          ptx::tma_load_2d_pair(a, &map_w, full0, kb * kMxStageBytes, n0);
          ptx::tma_load_2d_pair(a + kMxPairA, &map_x, full0, kb * kMxStageBytes, t0);
          ptx::tma_load_2d_pair(a + kMxPairA + kMxPairB, &map_ws, full0, kb * 256, n0 >> 7);
          ptx::tma_load_2d_pair(a + kMxPairA + kMxPairB + 2 * kMxTileBytes, &map_xs, full0, kb * 256, tile.t0 >> 7);
        }
        if (++stage == kMxPairStages) { stage = 0; phase ^= 1u; }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (rank == 0) {
      // ---------------------------------------------------------------- scales to tensor memory, products, for both CTAs
      const bool leader = ptx::elect_one();
      bool ok = true;
      int stage = 0, tiles = 0;
      uint32_t phase = 0;
      const uint32_t idesc0 = make_idesc_mxf4(256, kMxPairTokens, 0), idesc1 = make_idesc_mxf4(256, kMxPairTokens, 1);
      for (int u = pair; u < total && ok; u += pairs, ++tiles) {
        const uint32_t acc = tmem + (tiles & 1 ? kMxPairTokens : 0);
        // tokens of a tile may begin in the middle of a scale tile: 64 rows on are two columns on
        const uint32_t sb_shift = (static_cast<uint32_t>(mx_pair_tile(prm, u).t0) >> 5) & 3u;
        if (tiles > 1) {
          ok = mx_wait_hint(ptx::smem_u32(&sh->acc_free[tiles & 1]), static_cast<uint32_t>((tiles >> 1) - 1) & 1u, wait_limit, &sh->abort_flag, status);
          if (!ok) break;
          ptx::tc_fence_after();
        }
        for (int kb = 0; kb < prm.k_stages; ++kb) {
          const uint32_t full = ptx::smem_u32(&sh->full[stage]);
          if (wait_limit == 0u || !ptx::mbar_try_wait(full, phase)) {
            ok = mx_wait_hint(full, phase, wait_limit, &sh->abort_flag, status);
            if (!ok) break;
          }
          ptx::tc_fence_after();
          const uint32_t a = ring_addr + static_cast<uint32_t>(stage) * kMxPairStage;
          const uint64_t sa_desc = make_scale_desc(a + kMxPairA + kMxPairB), sb_desc = sa_desc + (2 * kMxTileBytes >> 4);
          const uint32_t sa = tmem + kMxPairScaleCol + static_cast<uint32_t>(stage) * kMxPairScaleCols, sb = sa + 8;
          const uint64_t a_desc = make_kmajor_desc(a, kMxStageBytes), b_desc = make_kmajor_desc(a + kMxPairA, kMxStageBytes);
          const bool both = prm.k_tiles - 2 * kb > 1;        // scale tiles of this stage: two but for an odd end
          if (leader) {
            ptx::tmem_copy_scales_pair(sa, sa_desc);
            ptx::tmem_copy_scales_pair(sb, sb_desc);
            ptx::tmem_copy_scales_pair(sb + 4, sb_desc + (2 * kMxTileBytes >> 4));
            if (both) {
              ptx::tmem_copy_scales_pair(sa + 4, sa_desc + (kMxTileBytes >> 4));
              ptx::tmem_copy_scales_pair(sb + 8, sb_desc + (kMxTileBytes >> 4));
              ptx::tmem_copy_scales_pair(sb + 12, sb_desc + (3 * kMxTileBytes >> 4));
            }
            ptx::mma_mxf4_pair(acc, a_desc, b_desc, idesc0, sa, sb + sb_shift, kb > 0);
            ptx::mma_mxf4_pair(acc, a_desc + 2, b_desc + 2, idesc1, sa, sb + sb_shift, 1u);
            if (both) {
              ptx::mma_mxf4_pair(acc, a_desc + 4, b_desc + 4, idesc0, sa + 4, sb + 8 + sb_shift, 1u);
              ptx::mma_mxf4_pair(acc, a_desc + 6, b_desc + 6, idesc1, sa + 4, sb + 8 + sb_shift, 1u);
            }
            ptx::mma_commit_pair(ptx::smem_u32(&sh->empty[stage]));
          }
          if (++stage == kMxPairStages) { stage = 0; phase ^= 1u; }
        }
        if (ok && leader) ptx::mma_commit_pair(ptx::smem_u32(&sh->acc_full[tiles & 1]));
      }
    }
    __syncwarp();
  } else {
    // -------------------------------------------------------------------- epilogue: lanes 32 (warp % 4) .., half the columns
    const int quad = warp & 3, half = (warp - 2) >> 2;
    const uint32_t free0 = ptx::map_to_cta(ptx::smem_u32(&sh->acc_free[0]), 0u);
    using Out = MxPairOut<Y>;
    const uint32_t my_out = ptx::smem_u32(out) + static_cast<uint32_t>(half) * Out::kBuffers * Out::kBufferBytes;
    const bool storer = quad == ((2 + 4 * half) & 3) && lane == 0;         // of this half
    int buffer = 0;
    int tiles = 0;
    for (int u = pair; u < total; u += pairs, ++tiles) {
      const MxPairTile tile = mx_pair_tile(prm, u);
      const int n0 = tile.n0 + static_cast<int>(rank) * 128, n = n0 + quad * 32 + lane;
      const float b = bias != nullptr && n < prm.N ? __ldg(bias + n) : 0.0f;
      const int buf = tiles & 1;
      const bool ok = mx_wait_hint(ptx::smem_u32(&sh->acc_full[buf]), static_cast<uint32_t>(tiles >> 1) & 1u, wait_limit, &sh->abort_flag, status);
      // (staged: the four warps of a half meet at barriers below, so they leave together)
      if (STAGED ? mx_half_vote(1 + half, !ok) : !__all_sync(0xffffffffu, ok)) break;
      ptx::tc_fence_after();
      const uint32_t lanes = tmem + (static_cast<uint32_t>(quad * 32) << 16) + (buf ? kMxPairTokens : 0) + half * (kMxPairTokens / 2);
      // All of the warp's columns first, then the accumulator is given back.  The arrival is a relaxed one: what it says is
      // that the reads above are complete (tcgen05.wait::ld), and no write of this thread has to be seen by whoever waits for
      // it; a release would wait for the stores of the tile before.  (By the memory model alone a relaxed arrival orders
      // nothing: this rests on the hardware, where reads that have been waited for are over and the next tile's MMAs start after the arrival.)
      uint32_t acc[kMxPairChunks][32];
#pragma unroll
      for (int k = 0; k < kMxPairChunks; ++k) ptx::tmem_ld_32x32(lanes + 32 * k, acc[k]);
      ptx::tmem_ld_wait();
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive_cluster_relaxed(free0 + 8u * static_cast<uint32_t>(buf));
      const int t0 = tile.t0 + half * (kMxPairTokens / 2);
      if constexpr (STAGED) {
#pragma unroll
        for (int k0 = 0; k0 < kMxPairChunks; k0 += Out::kBatch) {
          const uint32_t to = my_out + static_cast<uint32_t>(buffer) * Out::kBufferBytes;
          if (storer) ptx::bulk_wait_read<Out::kBuffers - 1>();            // the buffer's last stores have read it
          mx_half_sync(1 + half);
          const uint32_t mine = to + static_cast<uint32_t>(quad * 32 + lane) * sizeof(Y);
          if (prm.relu) mx_stage<Y, Out::kBatch, true>(mine, acc, k0, b); else mx_stage<Y, Out::kBatch, false>(mine, acc, k0, b);
          ptx::fence_async_smem();
          mx_half_sync(1 + half);
          if (storer) {
#pragma unroll
            for (int k = 0; k < Out::kBatch; ++k)
              if (n0 < prm.N && t0 + 32 * (k0 + k) < prm.T)
                ptx::tma_store_2d(&map_y, to + static_cast<uint32_t>(k) * Out::kChunkBytes, n0, t0 + 32 * (k0 + k));
            ptx::bulk_commit();                              // (also where nothing was stored: the waits count groups)
          }
          if (++buffer == Out::kBuffers) buffer = 0;
        }
      } else {
#pragma unroll
        for (int k = 0; k < kMxPairChunks; ++k)
          mx_store_column(acc[k], y + static_cast<size_t>(t0 + 32 * k) * prm.ld + n, prm.ld, n < prm.N ? prm.T - t0 - 32 * k : 0, b, prm.relu);
      }
    }
    if (STAGED && storer) ptx::bulk_wait_read<0>();           // shared memory stays until it has been read (the grid's end waits for the writes)
  }
  // Nothing of this CTA goes away while the peer can still signal its barriers or multiply into its tensor memory.
  ptx::tc_fence_before();
  __syncthreads();                                           // (no role of this CTA is still waiting: its flag is final)
  if (threadIdx.x == 0 && sh->abort_flag) ptx::st_cluster_u32(ptx::map_to_cta(ptx::smem_u32(const_cast<int*>(&sh->abort_flag)), rank ^ 1u), 1u);
  ptx::cluster_sync_all();                                   // (both CTAs know of a failure of either)
  if (sh->abort_flag) {
    // Any role of either CTA may have given up on work of others that had long issued it.  MMAs finish and copies land (in
    // microseconds; the barriers that count them need both CTAs' parts, which may not have been issued) before the memory of either goes away.
    if (warp == 1 && rank == 0 && ptx::elect_one()) {
      ptx::mma_commit_pair(ptx::smem_u32(&sh->drained));
      for (unsigned int i = 0; i < kDrainPolls && !ptx::mbar_try_wait_hint(ptx::smem_u32(&sh->drained), 0u); ++i) {}
    }
    if (threadIdx.x == 0)
      for (int i = 0; i < 256; ++i) __nanosleep(200);
    __syncthreads();
    ptx::cluster_sync_all();
  }
  if (warp == 1) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc_pair(tmem, kMxPairCols);
  }
}

}  // namespace qc
