// Products of microscaled 4-bit operands on the block-scaled tensor-core instruction (tcgen05.mma kind::mxf4, blocks of 32):
//   y[t][n] = relu?(bias[n] + sum over blocks b of 2^(sx[t][b] + sw[n][b] - 254) * sum over the block of cx cw),
// accumulated in 32 bits in tensor memory.  The weights are the instruction's M side (128 rows of a tile) and the tokens
// its N side (BN columns): a decoding step's few tokens then fill narrow columns, the epilogue's lanes
// hold neighbouring output channels of one token, so that plain stores are whole sectors whatever the sizes
// and alignments, and a channel's bias is one register.
//
// A ring stage is 256 values of the contraction (128 bytes a row, the 128-byte swizzle): weight and token codes by TMA in
// boxes of rows, their scales as tiles of 128 rows x 4 blocks (512 bytes; mx_format.cuh).  tcgen05.cp spreads a scale tile over
// four columns of tensor memory; the four instructions of a stage take two scales a row each out of them.  A ring
// stage has its own place there, so that the barrier that frees the stage also says that its scales have been read.
//
// Bound by the bytes of the weights up to about a hundred tokens (alone, in a captured graph: one token x 28672 x 8192 5.8 TB/s, 0.89
// of the measured copy rate; x 4096 x 4096 3.6 us, of which the launch is two thirds), then by filling shared memory.
//
// Roles (128 threads): warp 0 issues the loads, warp 1 owns tensor memory and issues copies and MMAs, then all four warps
// drain a quarter of the lanes each.  With few tiles a cluster of CTAs shares a tile: each takes a part of the contraction
// and sends its sums to the CTAs' shared memory, a share of the columns each, where they are added up in a fixed order (no
// scratch in global memory, and the same result each time).  All waits on mbarriers are bounded; why the cluster's own barriers
// and the allocation of tensor memory end is in tensor_memory.cuh.
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
__device__ __forceinline__ float4 lds_float4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
// The two halves of a cluster barrier.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
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
  static constexpr uint32_t kSA = 2 * kMxTileBytes, kSB = 2 * kMxTileBytes;
  static constexpr uint32_t kStage = kA + kB + kSA + kSB;              // a multiple of 1024
  static constexpr uint32_t kTx = kStage;
  static constexpr int kScaleCols = 16;                                // tensor-memory columns of a stage's scales
  // 256 columns of tensor memory for two CTAs an SM, 128 where four may run
  static constexpr int kCols = BN > 32 ? 256 : 128;
  static constexpr int kMaxStages = (kCols - BN) / kScaleCols < kMxMaxStages ? (kCols - BN) / kScaleCols : kMxMaxStages;
  static_assert(BN <= 128 && kMaxStages >= 2 && kStage % 1024 == 0);
};

// Stores a lane's sums of COUNT consecutive tokens (one channel, rows `ld` apart; the first `cols` count): bias, ReLU and
// rounding first, in place, then one store after the other from eight pointers.  A store reads its registers some tens of
// cycles after it was issued; with one value and one pointer that are made anew for each, a warp stores every 40 to 50 cycles.
template <int COUNT, typename Y>
__device__ __forceinline__ void mx_store_column(uint32_t (&acc)[COUNT], Y* y, size_t ld, int cols, float bias, bool relu) {
#pragma unroll
  for (int i = 0; i < COUNT; ++i) {
    float v = __uint_as_float(acc[i]) + bias;
    if (relu) v = v < 0.0f ? 0.0f : v;
    const Y r = from_float<Y>(v);
    if constexpr (sizeof(Y) == 4) acc[i] = __float_as_uint(v);
    else acc[i] = *reinterpret_cast<const unsigned short*>(&r);
  }
  Y* p[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) p[i] = y + i * ld;
#pragma unroll
  for (int i = 0; i < COUNT; ++i) {
    if (i < cols) {
      if constexpr (sizeof(Y) == 4) *reinterpret_cast<uint32_t*>(p[i & 7]) = acc[i];
      else *reinterpret_cast<unsigned short*>(p[i & 7]) = static_cast<unsigned short>(acc[i]);
    }
    p[i & 7] += 8 * ld;
  }
}

// Columns that a warp drains at a time.
template <int BN> constexpr int kMxChunk = BN < 32 ? 16 : 32;
template <int BN>
__device__ __forceinline__ void mx_drain(uint32_t taddr, uint32_t (&acc)[kMxChunk<BN>]) {
  if constexpr (kMxChunk<BN> == 16) ptx::tmem_ld_32x16(taddr, acc); else ptx::tmem_ld_32x32(taddr, acc);
  ptx::tmem_ld_wait();
}

// The sums of a tile shared by SPLIT CTAs (this one is number `part`; `cols` columns count, 0 after a failure).  Four columns
// at a time belong to CTA group % SPLIT: everyone's 128 x 4 sums go to that CTA's shared memory, 16 bytes a lane, and
// are added there in the order of the CTAs.  `done` gets each of this CTA's groups.
template <int SPLIT, int BN, typename Done>
__device__ __forceinline__ void mx_exchange(uint32_t lane_addr, uint32_t exchange_addr, int part, int cols, Done&& done) {
  constexpr uint32_t kPlace = 128 * 16;                      // bytes of a CTA's sums of a group
  const uint32_t mine = exchange_addr + threadIdx.x * 16;
  uint32_t to[SPLIT];
#pragma unroll
  for (int p = 0; p < SPLIT; ++p) to[p] = ptx::map_to_cta(mine + static_cast<uint32_t>(part) * kPlace, static_cast<uint32_t>(p));
  for (int c = 0; c < cols; c += kMxChunk<BN>) {             // (c / 4 is a multiple of SPLIT)
    uint32_t acc[kMxChunk<BN>];
    mx_drain<BN>(lane_addr + c, acc);
#pragma unroll
    for (int g = 0; g < kMxChunk<BN> / 4; ++g) {
      const uint32_t place = static_cast<uint32_t>((c / 4 + g) / SPLIT * SPLIT) * kPlace;
      if (c + 4 * g < cols) ptx::st_cluster_uint4(to[g % SPLIT] + place, acc[4 * g], acc[4 * g + 1], acc[4 * g + 2], acc[4 * g + 3]);
    }
  }
  ptx::cluster_sync_all();
  for (int g = part; 4 * g < cols; g += SPLIT) {
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int p = 0; p < SPLIT; ++p) {
      const float4 w = ptx::lds_float4(mine + static_cast<uint32_t>(g / SPLIT * SPLIT + p) * kPlace);
      v[0] += w.x; v[1] += w.y; v[2] += w.z; v[3] += w.w;
    }
    uint32_t bits[4] = {__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    done(4 * g, bits);
  }
}

template <int BN, typename Y>
__global__ void __launch_bounds__(kMxGemmThreads, 2)
mx_gemm_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x,
               const __grid_constant__ CUtensorMap map_ws, const __grid_constant__ CUtensorMap map_xs, const MxGemmParams prm,
               const float* __restrict__ bias, Y* __restrict__ y, int* status, unsigned int wait_limit) {
  using Tile = MxTile<BN>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  MxGemmShared* sh = reinterpret_cast<MxGemmShared*>(ring + static_cast<uint32_t>(prm.stages) * Tile::kStage);
  const uint32_t exchange_addr = (ptx::smem_u32(sh + 1) + 15u) & ~15u;   // split > 1: 128 sums of each column, or of 4 split columns
  const int warp = threadIdx.x >> 5;
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
  if (split > 1) ptx::cluster_arrive();
  ptx::grid_dependency_wait();                               // operands and y: other kernels' (the weights may be just written, too)
  ptx::grid_launch_dependents();

  // Both issuing warps run their loops with warp-uniform values, so that addresses, coordinates and descriptors live in
  // uniform registers, where copies and MMAs take their operands from; one lane issues.
  int issued = 0;                                            // stages loaded (warp 0)
  if (warp == 0) {
    // ------------------------------------------------------------------ loads
    const bool leader = ptx::elect_one();
    int stage = 0;
    uint32_t phase = 1;                                      // (the first pass over the ring finds every stage free)
    for (int kb = kb0; kb < kb1; ++kb, ++issued) {
      const uint32_t empty = ptx::smem_u32(&sh->empty[stage]);
      if (wait_limit == 0u || !ptx::mbar_try_wait(empty, phase)) {
        if (!mx_wait(empty, phase, wait_limit, &sh->abort_flag, status)) break;
      }
      const uint32_t bar = ptx::smem_u32(&sh->full[stage]);
      const uint32_t a = ring_addr + static_cast<uint32_t>(stage) * Tile::kStage;
      if (leader) {
        ptx::mbar_expect_tx(bar, Tile::kTx);
        ptx::tma_load_2d(a, &map_w, bar, kb * kMxStageBytes, n0);
        ptx::tma_load_2d(a + Tile::kA + Tile::kB, &map_ws, bar, kb * 256, tn);
        ptx::tma_load_2d(a + Tile::kA, &map_x, bar, kb * kMxStageBytes, t0);
        ptx::tma_load_2d(a + Tile::kA + Tile::kB + Tile::kSA, &map_xs, bar, kb * 256, t0 >> 7);
      }
      if (++stage == prm.stages) { stage = 0; phase ^= 1u; }
    }
    __syncwarp();
  } else if (warp == 1) {
    // ------------------------------------------------------------------ scales to tensor memory, products
    const bool leader = ptx::elect_one();
    int stage = 0;
    uint32_t phase = 0;
    const uint32_t idesc0 = make_idesc_mxf4(128, BN, 0), idesc1 = make_idesc_mxf4(128, BN, 1);
    for (int kb = kb0; kb < kb1; ++kb) {
      const uint32_t full = ptx::smem_u32(&sh->full[stage]);
      if (wait_limit == 0u || !ptx::mbar_try_wait(full, phase)) {
        if (!mx_wait(full, phase, wait_limit, &sh->abort_flag, status)) break;
      }
      ptx::tc_fence_after();
      const uint32_t a = ring_addr + static_cast<uint32_t>(stage) * Tile::kStage;
      const uint64_t sa_desc = make_scale_desc(a + Tile::kA + Tile::kB), sb_desc = sa_desc + (Tile::kSA >> 4);
      const uint32_t sa = tmem + BN + static_cast<uint32_t>(stage) * Tile::kScaleCols, sb = sa + 8;
      const uint64_t a_desc = make_kmajor_desc(a, kMxStageBytes), b_desc = make_kmajor_desc(a + Tile::kA, kMxStageBytes);
      const bool both = prm.k_tiles - 2 * kb > 1;            // scale tiles of this stage (128 values each): two but for an odd end
      if (leader) {
        ptx::tmem_copy_scales(sa, sa_desc);
        ptx::tmem_copy_scales(sb, sb_desc);
        if (both) {
          ptx::tmem_copy_scales(sa + 4, sa_desc + (kMxTileBytes >> 4));
          ptx::tmem_copy_scales(sb + 4, sb_desc + (kMxTileBytes >> 4));
        }
        ptx::mma_mxf4(tmem, a_desc, b_desc, idesc0, sa, sb, kb > kb0);
        ptx::mma_mxf4(tmem, a_desc + 2, b_desc + 2, idesc1, sa, sb, 1u);
        if (both) {
          ptx::mma_mxf4(tmem, a_desc + 4, b_desc + 4, idesc0, sa + 4, sb + 4, 1u);
          ptx::mma_mxf4(tmem, a_desc + 6, b_desc + 6, idesc1, sa + 4, sb + 4, 1u);
        }
        ptx::mma_commit(ptx::smem_u32(&sh->empty[stage]));
      }
      if (++stage == prm.stages) { stage = 0; phase ^= 1u; }
    }
    __syncwarp();
    if (leader) ptx::mma_commit(ptx::smem_u32(&sh->acc_full));            // (after a wait that expired: of what was issued)
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
  if (!good && warp == 0) {
    // The copies that were issued land before this CTA's shared memory goes away (bounded, whatever the caller's limit).  Any
    // role may have given up, also on copies of a loader that had long finished: so all of this comes after the flag is final.
    for (int i = 0; i < issued && i < prm.stages; ++i) {
      const int use = issued - 1 - i, s = use % prm.stages;
      const uint32_t parity = static_cast<uint32_t>(use / prm.stages) & 1u;
      for (unsigned int it = 0; it < kDrainPolls && !ptx::mbar_try_wait(ptx::smem_u32(&sh->full[s]), parity); ++it) {}
    }
    __syncwarp();
  }
  const int n = n0 + static_cast<int>(threadIdx.x);
  const uint32_t lane_addr = tmem + (static_cast<uint32_t>(warp * 32) << 16);
  const float b = bias != nullptr && n < prm.N ? __ldg(bias + n) : 0.0f;
  if (split == 1) {
    if (good)
      for (int c = 0; c < BN && t0 + c < prm.T; c += kMxChunk<BN>) {
        uint32_t acc[kMxChunk<BN>];
        mx_drain<BN>(lane_addr + c, acc);
        mx_store_column(acc, y + static_cast<size_t>(t0 + c) * prm.ld + n, prm.ld, n < prm.N ? prm.T - t0 - c : 0, b, prm.relu);
      }
  } else {
    ptx::cluster_wait();                                     // (the other CTAs run)
    auto sums = [&](int c, uint32_t (&v)[4]) {
      mx_store_column(v, y + static_cast<size_t>(t0 + c) * prm.ld + n, prm.ld, n < prm.N ? prm.T - t0 - c : 0, b, prm.relu);
    };
    const int cols = good ? min(BN, prm.T - t0) : 0;
    if (split == 2) mx_exchange<2, BN>(lane_addr, exchange_addr, part, cols, sums);
    else if (split == 4) mx_exchange<4, BN>(lane_addr, exchange_addr, part, cols, sums);
    else mx_exchange<8, BN>(lane_addr, exchange_addr, part, cols, sums);
  }
  ptx::tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem, Tile::kCols);
  }
}

}  // namespace qc
