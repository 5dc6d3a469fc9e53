// Quantized caches: the values of a token's heads are converted as they are written to their slot, and read back from
// any list of slots.  A head's D values are one group: int8 with an exponent for the group, or microscaled 4 bits.  Bound by
// HBM on long lists and by the launch on short ones: keys and values go in one launch, a head takes LANES lanes with V
// pieces of 32 bytes each, and a group of lanes has kCacheUnroll heads in flight and, on lists that the grid goes round more than
// once (75776 heads of 128 16-bit values), the slots of the next ones on their way (slot, then codes and scales, are dependent
// loads).  131072 tokens x 8 heads x 128 bf16, keys and values, int8: written in 141 us (0.88 of the measured copy rate), read back in
// 134 (0.93); in 4 bits 126 and 120 (0.83, 0.88).
#pragma once
#include "cache_items.cuh"
#include "mx_format.cuh"
#include "kernel_igemm.cuh"

namespace qc {

enum : int { CACHE_I8 = 0, CACHE_MX = 1 };
constexpr int kCacheThreads = 256;
constexpr int kCacheUnroll = 2, kCacheBlocks = 4;

struct CacheSide {
  uint8_t* codes;
  uint8_t* scales;
  void* values;              // written from or read into
  long long token, head;     // strides of `values`, in elements
};
struct CacheArgs {
  CacheSide side[2];         // keys, values
  const long long* slots;
  long long num_slots;
  int heads, D, blocks;
  int items;                 // rows * sides * heads, below 2^30
  FastDiv fd_heads;
  int sides;
  int unit;                  // bytes that heads of values may be reached in
  int lanes;                 // of a head, to be written
  int code_vec;              // a lane's int8 codes are aligned
  int code_pitch, scale_pitch;   // bytes of a head's codes and scales
};

struct CacheItem {
  bool valid, second;        // second: of the values, not the keys
  size_t values, group;      // element offset of the head's values; index of (slot, head)
};
__device__ __forceinline__ int cache_rows(const CacheArgs& a) { return a.items / (a.heads * a.sides); }
// The slot of item u (-1 behind the last); items are (row, side, head), head fastest.
__device__ __forceinline__ long long cache_slot(const CacheArgs& a, unsigned int u) {
  if (!cache_has(u, a.items)) return -1;
  int h;
  const int rs = a.fd_heads.divmod(static_cast<int>(u), &h), row = a.sides == 2 ? rs >> 1 : rs;
  return QC_IN(row, cache_rows(a)) ? __ldg(a.slots + row) : -1;
}
__device__ __forceinline__ CacheItem cache_item(const CacheArgs& a, unsigned int u, long long slot) {
  CacheItem c;
  int h;
  const int rs = a.fd_heads.divmod(static_cast<int>(u), &h);
  const int row = a.sides == 2 ? rs >> 1 : rs;
  c.second = a.sides == 2 && (rs & 1);
  c.valid = slot >= 0 && slot < a.num_slots;
  c.values = static_cast<size_t>(row * (c.second ? a.side[1].token : a.side[0].token) + h * (c.second ? a.side[1].head : a.side[0].head));
  c.group = static_cast<size_t>(slot) * a.heads + h;
  return c;
}
__device__ __forceinline__ uint8_t* cache_codes(const CacheArgs& a, const CacheItem& c) {
  return (c.second ? a.side[1].codes : a.side[0].codes) + c.group * a.code_pitch;
}
__device__ __forceinline__ uint8_t* cache_scales(const CacheArgs& a, const CacheItem& c) {
  return (c.second ? a.side[1].scales : a.side[0].scales) + c.group * a.scale_pitch;
}
// What those point into, for the checked build.
__device__ __forceinline__ Extent cache_codes_extent(const CacheArgs& a, const CacheItem& c) {
  return Extent::of(a.side[c.second].codes, static_cast<size_t>(a.num_slots) * a.heads * a.code_pitch);
}
__device__ __forceinline__ Extent cache_scales_extent(const CacheArgs& a, const CacheItem& c) {
  return Extent::of(a.side[c.second].scales, static_cast<size_t>(a.num_slots) * a.heads * a.scale_pitch);
}
template <typename T>
__device__ __forceinline__ Extent cache_values_extent(const CacheArgs& a, const CacheItem& c) {
  const CacheSide& s = a.side[c.second];
  return Extent::of(static_cast<const T*>(s.values), static_cast<size_t>((cache_rows(a) - 1) * s.token + (a.heads - 1) * s.head + a.D));
}
template <typename T>
__device__ __forceinline__ T* cache_values(const CacheArgs& a, const CacheItem& c) {
  return static_cast<T*>(c.second ? a.side[1].values : a.side[0].values) + c.values;
}

// How the lanes of a warp share out heads.  FEW: as few each as hold one, above LANES / 2, and the lanes behind the last
// whole group are idle.  Else LANES each.  (32768 tokens x 8 heads of bf16 to int8, few: 80 values 28.8 us, 96 33.8, 128
// 38.4; whole: 39.0, 39.4, 39.4.  Back, few: 30.5, 35.6, 40.9; whole: 32.5, 34.0, 36.3, so that reading has it whole.)
template <int LANES, bool FEW> struct CacheLanes {
  int G, per_warp, lane;
  unsigned int mine;             // which of the warp's heads; past all items where idle
  __device__ __forceinline__ CacheLanes(const CacheArgs& a) {
    const int l = threadIdx.x & 31;
    G = FEW ? a.lanes : LANES;
    per_warp = 32 / G;
    mine = cache_mine(l, G);
    lane = l % G;
  }
  // Maximum over a head's lanes: each looks 1, 2, 4, ... lanes ahead, around the group's end.
  __device__ __forceinline__ uint32_t max_over_head(uint32_t m) const {
    if constexpr (!FEW) {
      return max_over<LANES>(m);
    } else {
      const int first = (threadIdx.x & 31) - lane;
#pragma unroll
      for (int d = 1; d < LANES; d *= 2) m = max(m, __shfl_sync(0xffffffffu, m, first + (lane + d < G ? lane + d : lane + d - G)));
      return m;
    }
  }
};

// Up to LANES lanes a head, V pieces a lane.  ANY: values or int8 codes that a lane cannot reach by itself go through shared
// memory, in parts for LANES lanes.
template <typename T, int FMT, int LANES, int V, bool ANY>
__global__ void __launch_bounds__(kCacheThreads, V == 1 ? kCacheBlocks : 1)
cache_write_kernel(const CacheArgs a) {
  constexpr int E = Piece<T>::E, U = V == 1 ? kCacheUnroll : 1;
  __shared__ __align__(16) uint8_t stages[ANY ? kCacheThreads / 32 : 1][ANY ? kWarpStage : 1];
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const CacheLanes<LANES, !ANY> at(a);
  const unsigned int mine = at.mine;
  const int lane = at.lane, G = at.G, per_block = kCacheThreads / 32 * at.per_warp, step = gridDim.x * per_block;
  uint8_t* stage = stages[ANY ? threadIdx.x >> 5 : 0];
  // the lanes of a warp run the same number of rounds
  const int warp_first = (threadIdx.x >> 5) * at.per_warp;
  long long slot[U];
#pragma unroll
  for (int j = 0; j < U; ++j) slot[j] = cache_slot(a, cache_unit(blockIdx.x * per_block + warp_first + j * step, mine));
  for (int base = blockIdx.x * per_block + warp_first; base < a.items; base += U * step) {
    CacheItem c[U];
    Piece<T> x[U][V];
#pragma unroll
    for (int j = 0; j < U; ++j) c[j] = cache_item(a, cache_unit(base + j * step, mine), slot[j]);
#pragma unroll
    for (int j = 0; j < U; ++j) slot[j] = cache_slot(a, cache_unit(base + (U + j) * step, mine));
#pragma unroll
    for (int j = 0; j < U; ++j)
#pragma unroll
      for (int k = 0; k < V; ++k)
        group_load<ANY>(x[j][k], cache_values<T>(a, c[j]) + k * G * E, c[j].valid ? a.D - k * G * E : 0, G, lane, a.unit, stage,
                        cache_values_extent<T>(a, c[j]));
#pragma unroll
    for (int j = 0; j < U; ++j) {
      uint8_t* codes = cache_codes(a, c[j]);
      uint8_t* scales = cache_scales(a, c[j]);
      const Extent of_codes = cache_codes_extent(a, c[j]), of_scales = cache_scales_extent(a, c[j]);
      if constexpr (FMT == CACHE_I8) {
        float v[V][E];
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < V; ++k) {
          x[j][k].unpack(v[k]);
          m = max(m, finite_top<1>(v[k], x[j][k].top()));
        }
        const uint32_t sb = i8_scale_byte(at.max_over_head(m));
        const float inv = inverse_scale(sb);
        if (c[j].valid && lane == 0 && QC_AT(of_scales, scales, 1)) *scales = static_cast<uint8_t>(sb);
#pragma unroll
        for (int k = 0; k < V; ++k) {
          const int first = k * G * E, n = c[j].valid ? min(a.D - first, G * E) : 0;
          uint32_t w[E / 4];
#pragma unroll
          for (int i = 0; i < E / 4; ++i) w[i] = i8_encode_four(v[k] + 4 * i, inv);
          if constexpr (ANY) {
            uint8_t* group = stage + ((threadIdx.x & 31) - lane) * E;
#pragma unroll
            for (int i = 0; i < E / 4; ++i) reinterpret_cast<uint32_t*>(group)[lane * (E / 4) + i] = w[i];
            __syncwarp();
            store_bytes<E>(codes + first, group, n, G, lane, of_codes);
            __syncwarp();
          } else if (lane * E < n && QC_AT(of_codes, codes + first + lane * E, E)) {
            if constexpr (E == 8) *reinterpret_cast<uint2*>(codes + first + lane * E) = make_uint2(w[0], w[1]);
            else *reinterpret_cast<uint4*>(codes + first + lane * E) = make_uint4(w[0], w[1], w[2], w[3]);
          }
        }
      } else {
        constexpr int kBlockLanes = kMxBlock / E;
#pragma unroll
        for (int k = 0; k < V; ++k) {
          const int col = (k * G + lane) * E;
          float v[E];
          x[j][k].unpack(v);
          const uint32_t sb = mx_scale_byte(finite_top<kBlockLanes>(v, x[j][k].top()), kCoverRoundUp);
          if (!c[j].valid || col >= a.blocks * kMxBlock) continue;
          mx_store_codes(codes + col / 2, v, inverse_scale(sb), of_codes);
          if ((col & (kMxBlock - 1)) == 0 && QC_AT(of_scales, scales + col / kMxBlock, 1)) scales[col / kMxBlock] = static_cast<uint8_t>(sb);
        }
      }
    }
  }
}

template <typename T, int FMT, int LANES, int V, bool ANY>
__global__ void __launch_bounds__(kCacheThreads, V == 1 ? kCacheBlocks : 1)
cache_read_kernel(const CacheArgs a) {
  constexpr int E = Piece<T>::E, U = V == 1 ? kCacheUnroll : 1;
  __shared__ __align__(16) uint8_t stages[ANY ? kCacheThreads / 32 : 1][ANY ? kWarpStage : 1];
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  constexpr int kPerWarp = 32 / LANES, kPerBlock = kCacheThreads / LANES;
  const int lane = threadIdx.x & (LANES - 1);
  const int step = gridDim.x * kPerBlock;
  uint8_t* stage = stages[ANY ? threadIdx.x >> 5 : 0];
  const int warp_first = (threadIdx.x >> 5) * kPerWarp;
  const unsigned int mine = cache_mine(threadIdx.x & 31, LANES);
  long long slot[U];
#pragma unroll
  for (int j = 0; j < U; ++j) slot[j] = cache_slot(a, cache_unit(blockIdx.x * kPerBlock + warp_first + j * step, mine));
  for (int base = blockIdx.x * kPerBlock + warp_first; base < a.items; base += U * step) {
    CacheItem c[U];
    uint32_t w[U][V][E / 4], sb[U][V];                      // (4-bit codes: the first half)
    DealtBytes<E> raw[FMT == CACHE_I8 && ANY ? U : 1][V];
#pragma unroll
    for (int j = 0; j < U; ++j) c[j] = cache_item(a, cache_unit(base + j * step, mine), slot[j]);
#pragma unroll
    for (int j = 0; j < U; ++j) slot[j] = cache_slot(a, cache_unit(base + (U + j) * step, mine));
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const uint8_t* codes = cache_codes(a, c[j]);
      const uint8_t* scales = cache_scales(a, c[j]);
      const Extent of_codes = cache_codes_extent(a, c[j]), of_scales = cache_scales_extent(a, c[j]);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const int col = (k * LANES + lane) * E, n = c[j].valid ? min(E, a.D - col) : 0;
#pragma unroll
        for (int i = 0; i < E / 4; ++i) w[j][k][i] = 0u;
        sb[j][k] = kScaleOne;
        if constexpr (FMT == CACHE_I8 && ANY)
          load_bytes<E>(raw[j][k], codes + k * LANES * E, c[j].valid ? min(a.D - k * LANES * E, LANES * E) : 0, LANES, lane, of_codes);
        if (n <= 0) continue;
        if constexpr (FMT == CACHE_I8) {
          if (QC_AT(of_scales, scales, 1)) sb[j][k] = __ldg(scales);
          if constexpr (!ANY) {
            if (!QC_AT(of_codes, codes + col, n)) continue;
            if (a.code_vec) {
              if constexpr (E == 8) {
                const uint2 q = __ldg(reinterpret_cast<const uint2*>(codes + col));
                w[j][k][0] = q.x; w[j][k][1] = q.y;
              } else {
                const uint4 q = __ldg(reinterpret_cast<const uint4*>(codes + col));
                w[j][k][0] = q.x; w[j][k][1] = q.y; w[j][k][2] = q.z; w[j][k][3] = q.w;
              }
            } else {
#pragma unroll
              for (int i = 0; i < E; ++i)
                if (i < n) w[j][k][i / 4] |= static_cast<uint32_t>(__ldg(codes + col + i)) << (8 * (i & 3));
            }
          }
        } else {
          if (!QC_AT(of_scales, scales + col / kMxBlock, 1) || !QC_AT(of_codes, codes + col / 2, E / 2)) continue;
          sb[j][k] = __ldg(scales + col / kMxBlock);
          if constexpr (E == 8) {
            w[j][k][0] = __ldg(reinterpret_cast<const uint32_t*>(codes + col / 2));
          } else {
            const uint2 q = __ldg(reinterpret_cast<const uint2*>(codes + col / 2));
            w[j][k][0] = q.x; w[j][k][1] = q.y;
          }
        }
      }
    }
#pragma unroll
    for (int j = 0; j < U; ++j) {
      T* y = cache_values<T>(a, c[j]);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        float v[E];
        const float scale = scale_of(sb[j][k]);
        if constexpr (FMT == CACHE_I8 && ANY)
          gather_bytes<E>(w[j][k], raw[j][k], cache_codes(a, c[j]) + k * LANES * E, c[j].valid ? min(a.D - k * LANES * E, LANES * E) : 0, LANES, lane,
                          stage);
        if constexpr (FMT == CACHE_I8) {
#pragma unroll
          for (int i = 0; i < E / 4; ++i) i8_decode_four(w[j][k][i], scale, v + 4 * i);
        } else {
#pragma unroll
          for (int i = 0; i < E / 8; ++i) mx_decode_eight(w[j][k][i], scale, v + 8 * i);
        }
        Piece<T> p;
        p.pack(v);
        group_store<ANY>(p, y + k * LANES * E, c[j].valid ? a.D - k * LANES * E : 0, LANES, lane, a.unit, stage,
                         cache_values_extent<T>(a, c[j]));
      }
    }
  }
}

}  // namespace qc
