// Quantized caches: the values of a token's heads are converted as they are written to their slot, and read back from
// any list of slots.  A head's D values are one group: int8 with an exponent for the group, or microscaled 4 bits.  Bound by
// HBM on long lists and by the launch on short ones: keys and values go in one launch, a head takes 8, 16 or 32 lanes
// with eight values a lane (several times over where D > 256).
#pragma once
#include "mx_format.cuh"
#include "kernel_igemm.cuh"

namespace qc {

enum : int { CACHE_I8 = 0, CACHE_MX = 1 };
constexpr int kCacheThreads = 256;

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
  int vec_ok, code_vec;      // eight values / eight int8 codes are aligned
  int code_pitch, scale_pitch;   // bytes of a head's codes and scales
};

struct CacheItem {
  int side;
  bool valid;
  size_t values, group;      // element offset of the head's values; index of (slot, head)
};
__device__ __forceinline__ CacheItem cache_item(const CacheArgs& a, int u) {
  CacheItem c = {0, false, 0, 0};
  if (u >= a.items) return c;
  int h;
  const int rs = a.fd_heads.divmod(u, &h);
  const int row = a.sides == 2 ? rs >> 1 : rs;
  c.side = a.sides == 2 ? rs & 1 : 0;
  const long long slot = __ldg(a.slots + row);
  c.valid = slot >= 0 && slot < a.num_slots;
  const CacheSide& s = a.side[c.side];
  c.values = static_cast<size_t>(row * s.token + h * s.head);
  c.group = static_cast<size_t>(slot) * a.heads + h;
  return c;
}

// LANES lanes a head, V vectors of eight values a lane.
template <typename T, int FMT, int LANES, int V>
__global__ void __launch_bounds__(kCacheThreads)
cache_write_kernel(const CacheArgs a) {
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  constexpr int kPerBlock = kCacheThreads / LANES;
  const int lane = threadIdx.x & (LANES - 1);
  const int step = gridDim.x * kPerBlock;
  // the lanes of a warp run the same number of rounds
  const int mine = threadIdx.x / LANES, warp_first = (threadIdx.x & ~31) / LANES;
  for (int base = blockIdx.x * kPerBlock + warp_first; base < a.items; base += step) {
    const CacheItem c = cache_item(a, base + mine - warp_first);
    const CacheSide& s = a.side[c.side];
    const T* x = static_cast<const T*>(s.values) + c.values;
    float v[V][8];
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const int col = (k * LANES + lane) * 8, n = a.D - col;
      if (c.valid && n >= 8 && a.vec_ok) {
        Eight<T> e;
        e.load(x + col);
        e.unpack(v[k]);
      } else {
        load_some(x + col, c.valid ? n : 0, v[k]);
      }
    }
    uint8_t* codes = s.codes + c.group * a.code_pitch;
    uint8_t* scales = s.scales + c.group * a.scale_pitch;
    const bool in = c.valid && QC_IN(c.group, static_cast<size_t>(a.num_slots) * a.heads);
    if constexpr (FMT == CACHE_I8) {
      uint32_t m = 0;
#pragma unroll
      for (int k = 0; k < V; ++k) m = max(m, finite_top<1>(v[k]));
      const uint32_t sb = i8_scale_byte(max_over<LANES>(m));
      if (in && lane == 0) *scales = static_cast<uint8_t>(sb);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const int col = (k * LANES + lane) * 8, n = min(8, a.D - col);
        if (!in || n <= 0) continue;
        const uint2 w = i8_encode_eight(v[k], inverse_scale(sb));
        if (n == 8 && a.code_vec) *reinterpret_cast<uint2*>(codes + col) = w;
        else
          for (int i = 0; i < n; ++i) codes[col + i] = static_cast<uint8_t>((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
      }
    } else {
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const int col = (k * LANES + lane) * 8;
        const uint32_t sb = mx_scale_byte(finite_top<4>(v[k]), 0x3FFFFFu);
        if (!in || col >= a.blocks * kMxBlock) continue;
        *reinterpret_cast<uint32_t*>(codes + col / 2) = mx_encode_eight(v[k], inverse_scale(sb));
        if ((col & 31) == 0) scales[col / kMxBlock] = static_cast<uint8_t>(sb);
      }
    }
  }
}

constexpr int kCacheUnroll = 4;                 // heads a group of lanes has in flight on the way back

template <typename T, int FMT, int LANES, int V>
__global__ void __launch_bounds__(kCacheThreads)
cache_read_kernel(const CacheArgs a) {
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  constexpr int kPerBlock = kCacheThreads / LANES;
  constexpr int U = V == 1 ? kCacheUnroll : 1;
  const int lane = threadIdx.x & (LANES - 1);
  const int step = gridDim.x * kPerBlock;
  for (int base = blockIdx.x * kPerBlock + threadIdx.x / LANES; base < a.items; base += U * step) {
    CacheItem c[U];
    uint2 w[U][V];
    uint32_t sb[U][V];
#pragma unroll
    for (int j = 0; j < U; ++j) c[j] = cache_item(a, base + j * step);
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const uint8_t* codes = a.side[c[j].side].codes + c[j].group * a.code_pitch;
      const uint8_t* scales = a.side[c[j].side].scales + c[j].group * a.scale_pitch;
      const bool in = c[j].valid && QC_IN(c[j].group, static_cast<size_t>(a.num_slots) * a.heads);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const int col = (k * LANES + lane) * 8, n = min(8, a.D - col);
        w[j][k] = make_uint2(0u, 0u);
        sb[j][k] = kScaleOne;
        if (!in || n <= 0) continue;
        if constexpr (FMT == CACHE_I8) {
          sb[j][k] = __ldg(scales);
          if (n == 8 && a.code_vec) w[j][k] = __ldg(reinterpret_cast<const uint2*>(codes + col));
          else
            for (int i = 0; i < n; ++i) {
              const uint32_t b = static_cast<uint32_t>(__ldg(codes + col + i)) << (8 * (i & 3));
              if (i < 4) w[j][k].x |= b; else w[j][k].y |= b;
            }
        } else {
          sb[j][k] = __ldg(scales + col / kMxBlock);
          w[j][k].x = __ldg(reinterpret_cast<const uint32_t*>(codes + col / 2));
        }
      }
    }
#pragma unroll
    for (int j = 0; j < U; ++j) {
      if (!c[j].valid) continue;
      T* y = static_cast<T*>(a.side[c[j].side].values) + c[j].values;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const int col = (k * LANES + lane) * 8, n = a.D - col;
        if (n <= 0) continue;
        float v[8];
        if constexpr (FMT == CACHE_I8) i8_decode_eight(w[j][k], scale_of(sb[j][k]), v);
        else mx_decode_eight(w[j][k].x, scale_of(sb[j][k]), v);
        if (n >= 8 && a.vec_ok) {
          Eight<T> e;
          e.pack(v);
          e.store(y + col);
        } else {
          store_some(y + col, n, v);
        }
      }
    }
  }
}

}  // namespace qc
