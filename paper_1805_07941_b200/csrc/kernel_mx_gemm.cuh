// Products of microscaled 4-bit operands on the block-scaled tensor-core instruction (tcgen05.mma kind::mxf4, blocks of 32):
//   y[t][n] = relu?(bias[n] + sum over blocks b of 2^(sx[t][b] + sw[n][b] - 254) * sum over the block of cx cw),
// accumulated in 32 bits in tensor memory.  The weights are the instruction's M side (128 rows of a tile) and the tokens
// its N side (BN columns): a decoding step's few tokens then fill narrow columns, the epilogue's lanes
// hold neighbouring output channels of one token, so that plain stores are whole sectors whatever the sizes
// and alignments, and a channel's bias is one register.
//
// A ring stage is 256 values of the contraction (128 bytes a row, the 128-byte swizzle): weight and token codes by TMA in
// boxes of rows, their scales as tiles of 128 rows x 4 blocks (512 bytes; mx_format.cuh).  tcgen05.cp spreads a scale tile over
// four columns of tensor memory; the four instructions of a stage take two scales a row each out of them.  The scales
// have two places in tensor memory, and a stage's copies wait until the instructions that read the place
// two stages before have finished.
//
// Roles (128 threads): warp 0 issues the loads, warp 1 owns tensor memory and issues copies and MMAs, then all four warps
// drain a quarter of the lanes each.  With few tiles a cluster of CTAs shares a tile: each takes a part of the contraction,
// leaves its sums in shared memory, and adds up its share of the columns over the cluster in a fixed order (no
// scratch in global memory, and the same result each time).  All waits are bounded.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <cstdint>
#include "kernel_igemm.cuh"
#include "mx_format.cuh"

namespace qc {

constexpr int kMxStageBytes = 128;              // bytes of a row's codes in a stage: 256 values
constexpr int kMxMaxStages = 8;
constexpr int kMxGemmThreads = 128;

struct MxGemmParams {
  int N, T;                        // output channels, tokens
  int tiles_n, tiles_t;
  int k_stages;                    // ceil(K / 256)
  int k_tiles;                     // scale tiles along the contraction, ceil(K / 128)
  int stages;                      // of the ring
  int split;                       // CTAs of a cluster that share a tile
  int relu;
  uint32_t ring_bytes;             // of the ring, or of the sums that a cluster's CTAs leave in it if those need more
  size_t ld;                       // of y, in elements
};

struct MxGemmShared {
  uint64_t full[kMxMaxStages];
  uint64_t empty[kMxMaxStages];
  uint64_t acc_full;
  uint32_t tmem_base;
  volatile int abort_flag;
};

namespace ptx {
__device__ __forceinline__ void mma_mxf4(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t sa_tmem,
                                         uint32_t sb_tmem, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
      ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sa_tmem), "r"(sb_tmem), "r"(accumulate)
      : "memory");
}
// 32 rows of 16 bytes in shared memory to four columns of tensor memory, the same in each of the four lane quarters.
__device__ __forceinline__ void tmem_copy_scales(uint32_t taddr, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
__device__ __forceinline__ float ld_cluster_f32(uint32_t cluster_addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(cluster_addr) : "memory");
  return v;
}
__device__ __forceinline__ void sts_f32(uint32_t addr, float v) {
  asm volatile("st.shared.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}
}  // namespace ptx

// Shared-memory descriptor of a scale tile: 32 rows of 16 bytes, no swizzle, groups of eight rows 128 bytes apart.
__device__ __forceinline__ uint64_t make_scale_desc(uint32_t smem_addr) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((smem_addr >> 4) & 0x3FFFu);
  d |= static_cast<uint64_t>(128u >> 4) << 32;
  d |= 1ull << 46;
  return d;
}
// Instruction descriptor: 4-bit operands (2 exponent bits, 1 significand bit), scales of 8 exponent bits, K-major, M rows,
// N = bn; `half`: which two of a word's four scales.
__device__ __forceinline__ uint32_t make_idesc_mxf4(int m, int bn, uint32_t half) {
  uint32_t d = 0;
  d |= (2u * half) << 4;                         // first scale of B in its word
  d |= 1u << 7;                                  // A: E2M1
  d |= 1u << 10;                                 // B: E2M1
  d |= static_cast<uint32_t>(bn >> 3) << 17;
  d |= 1u << 23;                                 // scales: UE8M0
  d |= static_cast<uint32_t>(m >> 4) << 24;
  d |= (2u * half) << 29;                        // first scale of A in its word
  return d;
}

// Bounded wait of this kernel's roles: false (with the block's abort flag and the status raised) once the limit is used up,
// or when another role gave up.
__device__ __forceinline__ bool mx_wait(uint32_t bar, uint32_t parity, unsigned int limit, volatile int* abort_flag, int* status) {
  for (unsigned int it = 0; it < limit; ++it) {
    if (ptx::mbar_try_wait(bar, parity)) return true;
    if (*abort_flag) return false;
  }
  *abort_flag = 1;
  atomicExch(status, kStatusTimeout);
  return false;
}

template <int BN> struct MxTile {
  static constexpr uint32_t kA = 128 * kMxStageBytes, kB = BN * kMxStageBytes;
  static constexpr int kTileAtomsB = (BN + 127) / 128;
  static constexpr uint32_t kSA = 2 * kMxTileBytes, kSB = 2 * kTileAtomsB * kMxTileBytes;
  static constexpr uint32_t kStage = kA + kB + kSA + kSB;              // a multiple of 1024
  static constexpr uint32_t kTx = kStage;
  static constexpr int kScaleCols = 8 + 8 * kTileAtomsB;               // tensor-memory columns of a stage's scales
  static constexpr int kUsedCols = BN + 2 * kScaleCols;
  static constexpr int kCols = kUsedCols <= 64 ? 64 : kUsedCols <= 128 ? 128 : kUsedCols <= 256 ? 256 : 512;
  static_assert(kUsedCols <= 512 && kStage % 1024 == 0);
};

template <int BN, typename Y>
__global__ void __launch_bounds__(kMxGemmThreads)
mx_gemm_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x,
               const __grid_constant__ CUtensorMap map_ws, const __grid_constant__ CUtensorMap map_xs, const MxGemmParams prm,
               const float* __restrict__ bias, Y* __restrict__ y, int* status, unsigned int wait_limit) {
  using Tile = MxTile<BN>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  MxGemmShared* sh = reinterpret_cast<MxGemmShared*>(ring + prm.ring_bytes);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int split = prm.split;
  const int part = split > 1 ? static_cast<int>(ptx::cluster_ctarank()) : 0;
  const int tile = static_cast<int>(blockIdx.x) / split;
  const int tt = tile / prm.tiles_n, tn = tile - tt * prm.tiles_n;
  const int n0 = tn * 128, t0 = tt * BN;
  // this CTA's stages of the contraction (at least one each: the host keeps split <= k_stages)
  const int kb0 = static_cast<int>(static_cast<long long>(prm.k_stages) * part / split);
  const int kb1 = static_cast<int>(static_cast<long long>(prm.k_stages) * (part + 1) / split);
  const uint32_t ring_addr = ptx::smem_u32(ring);

  if (threadIdx.x == 0) {
    for (int s = 0; s < prm.stages; ++s) {
      ptx::mbar_init(ptx::smem_u32(&sh->full[s]), 1);
      ptx::mbar_init(ptx::smem_u32(&sh->empty[s]), 1);
    }
    ptx::mbar_init(ptx::smem_u32(&sh->acc_full), 1);
    sh->abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    ptx::fence_async_smem();
    ptx::prefetch_tmap(&map_w);
    ptx::prefetch_tmap(&map_x);
    ptx::prefetch_tmap(&map_ws);
    ptx::prefetch_tmap(&map_xs);
  }
  if (warp == 1) {
    ptx::tmem_alloc(ptx::smem_u32(&sh->tmem_base), Tile::kCols);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = sh->tmem_base;
  ptx::grid_dependency_wait();                               // operands and y: other kernels' (the weights may be just written, too)
  ptx::grid_launch_dependents();

  if (warp == 0) {
    if (lane == 0) {
      // ---------------------------------------------------------------- loads
      bool ok = true;
      int stage = 0, issued = 0;
      uint32_t phase = 0;
      for (int kb = kb0; kb < kb1 && ok; ++kb, ++issued) {
        if (issued >= prm.stages) {
          ok = mx_wait(ptx::smem_u32(&sh->empty[stage]), phase ^ 1u, wait_limit, &sh->abort_flag, status);
          if (!ok) break;
        }
        const uint32_t bar = ptx::smem_u32(&sh->full[stage]);
        const uint32_t a = ring_addr + static_cast<uint32_t>(stage) * Tile::kStage;
        ptx::mbar_expect_tx(bar, Tile::kTx);
        ptx::tma_load_2d(a, &map_w, bar, kb * kMxStageBytes, n0);
        ptx::tma_load_2d(a + Tile::kA + Tile::kB, &map_ws, bar, kb * 256, tn);
        ptx::tma_load_2d(a + Tile::kA, &map_x, bar, kb * kMxStageBytes, t0);
        ptx::tma_load_2d(a + Tile::kA + Tile::kB + Tile::kSA, &map_xs, bar, kb * 256, t0 >> 7);
        if (++stage == prm.stages) { stage = 0; phase ^= 1u; }
      }
      if (!ok || sh->abort_flag) {
        // the copies already issued land before this CTA's shared memory goes away (bounded, whatever the caller's limit)
        for (int i = 0; i < issued && i < prm.stages; ++i) {
          const int use = issued - 1 - i, s = use % prm.stages;
          const uint32_t parity = static_cast<uint32_t>(use / prm.stages) & 1u;
          for (unsigned int it = 0; it < kDrainPolls && !ptx::mbar_try_wait(ptx::smem_u32(&sh->full[s]), parity); ++it) {}
        }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0) {
      // ---------------------------------------------------------------- scales to tensor memory, products
      bool ok = true;
      int stage = 0;
      uint32_t phase = 0;
      const uint32_t idesc0 = make_idesc_mxf4(128, BN, 0), idesc1 = make_idesc_mxf4(128, BN, 1);
      for (int kb = kb0, it = 0; kb < kb1; ++kb, ++it) {
        ok = mx_wait(ptx::smem_u32(&sh->full[stage]), phase, wait_limit, &sh->abort_flag, status);
        if (ok && it >= 2) {
          // the instructions of two stages ago have read their scales out of the place that this stage's go to
          const int use = it - 2, s = use % prm.stages;
          ok = mx_wait(ptx::smem_u32(&sh->empty[s]), static_cast<uint32_t>(use / prm.stages) & 1u, wait_limit, &sh->abort_flag, status);
        }
        if (!ok) break;
        ptx::tc_fence_after();
        const uint32_t a = ring_addr + static_cast<uint32_t>(stage) * Tile::kStage;
        const uint32_t sa_smem = a + Tile::kA + Tile::kB, sb_smem = sa_smem + Tile::kSA;
        const uint32_t sa = tmem + BN + static_cast<uint32_t>(it & 1) * Tile::kScaleCols, sb = sa + 8;
        const uint64_t a_desc = make_kmajor_desc(a, kMxStageBytes), b_desc = make_kmajor_desc(a + Tile::kA, kMxStageBytes);
        const int halves = min(2, prm.k_tiles - 2 * kb);     // scale tiles of this stage: 128 values each
        for (int k = 0; k < halves; ++k) {
          ptx::tmem_copy_scales(sa + 4 * k, make_scale_desc(sa_smem + k * kMxTileBytes));
#pragma unroll
          for (int j = 0; j < Tile::kTileAtomsB; ++j)
            ptx::tmem_copy_scales(sb + 4 * (k * Tile::kTileAtomsB + j), make_scale_desc(sb_smem + (2 * j + k) * kMxTileBytes));
          const uint32_t sbk = sb + 4 * k * Tile::kTileAtomsB;
          ptx::mma_mxf4(tmem, a_desc + 4 * k, b_desc + 4 * k, idesc0, sa + 4 * k, sbk, it > 0 || k > 0);
          ptx::mma_mxf4(tmem, a_desc + 4 * k + 2, b_desc + 4 * k + 2, idesc1, sa + 4 * k, sbk, 1u);
        }
        ptx::mma_commit(ptx::smem_u32(&sh->empty[stage]));
        if (++stage == prm.stages) { stage = 0; phase ^= 1u; }
      }
      ptx::mma_commit(ptx::smem_u32(&sh->acc_full));          // (after a wait that expired: of what was issued)
    }
    __syncwarp();
  }
  // -------------------------------------------------------------------- epilogue: warp w drains lanes 32 w .. 32 w + 31
  // The barrier of the products is waited for in any case: nothing of this CTA goes away under a running instruction.
  bool done = false;
  for (unsigned int it = 0; it < kDrainPolls && !done; ++it) done = ptx::mbar_try_wait_hint(ptx::smem_u32(&sh->acc_full), 0u) != 0;
  if (!done) { sh->abort_flag = 1; atomicExch(status, kStatusTimeout); }
  __syncthreads();                                           // (no role is still waiting: the flag is final)
  ptx::tc_fence_after();
  const bool good = sh->abort_flag == 0;
  const int n = n0 + static_cast<int>(threadIdx.x);
  const uint32_t lane_addr = tmem + (static_cast<uint32_t>(warp * 32) << 16);
  const float b = bias != nullptr && n < prm.N ? __ldg(bias + n) : 0.0f;
  auto store = [&](int t, float v) {
    v += b;
    if (prm.relu) v = v < 0.0f ? 0.0f : v;
    if (t < prm.T && n < prm.N) y[static_cast<size_t>(t) * prm.ld + n] = from_float<Y>(v);
  };
  constexpr int kChunk = BN < 32 ? 16 : 32;
  if (split == 1) {
    if (good)
      for (int c = 0; c < BN && t0 + c < prm.T; c += kChunk) {
        uint32_t acc[kChunk];
        if constexpr (kChunk == 16) ptx::tmem_ld_32x16(lane_addr + c, acc); else ptx::tmem_ld_32x32(lane_addr + c, acc);
        ptx::tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < kChunk; ++i) store(t0 + c + i, __uint_as_float(acc[i]));
      }
  } else {
    // columns of 128 sums each, in the ring's memory: its loads and the instructions that read them are done
    const int cols = min(BN, prm.T - t0);
    if (good)
      for (int c = 0; c < cols; c += kChunk) {
        uint32_t acc[kChunk];
        if constexpr (kChunk == 16) ptx::tmem_ld_32x16(lane_addr + c, acc); else ptx::tmem_ld_32x32(lane_addr + c, acc);
        ptx::tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < kChunk; ++i)
          ptx::sts_f32(ring_addr + static_cast<uint32_t>((c + i) * 128 + threadIdx.x) * 4, __uint_as_float(acc[i]));
      }
    ptx::cluster_sync_all();
    for (int c = part; c < cols; c += split) {
      const uint32_t at = ring_addr + static_cast<uint32_t>(c * 128 + threadIdx.x) * 4;
      float v = 0.0f;
      for (int p = 0; p < split; ++p) v += ptx::ld_cluster_f32(ptx::map_to_cta(at, static_cast<uint32_t>(p)));
      store(t0 + c, v);
    }
    ptx::cluster_sync_all();                                 // the others may still read this CTA's sums
  }
  ptx::tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem, Tile::kCols);
  }
}

}  // namespace qc
