// Microscaled 4-bit values: the (4, 1) type of Section 2.1 in blocks of 32 along a row, each block with a scale alpha = 2^e
// of its own.  A code is the sign-and-magnitude pattern of Eq. 2 (bit 3 the sign, then two exponent bits, then one
// significand bit); here its value is taken in halves, so that the magnitudes are 0, 1/2, 1, 3/2, 2, 3, 4, 6 (Eq. 2's integers
// 0, 1, 2, 3, 4, 6, 8, 12 divided by 2), as the tensor cores read them.  A block's scale is one byte s = e + 127.
//
// Layouts: two codes to a byte, the even-numbered one in the low half, a row padded with zero codes to whole blocks (16
// bytes each).  Scale bytes either lie row by row, or in tiles of 128 rows x 4 blocks, 512 bytes each, tile (r / 128, b / 4)
// after tile along the row: byte (r % 32) * 16 + (r % 128 / 32) * 4 + b % 4 of a tile.  That is the order in which
// tcgen05.cp spreads them over tensor memory (32 lanes x 16 bytes), so that a product needs no reordering, and the four
// scales of 128 consecutive values are one word.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <cstdint>
#include <cstring>
#include <type_traits>

#include "epilogue.cuh"
#include "extent.cuh"

namespace qc {

constexpr int kMxBlock = 32;                    // values to a scale
constexpr int kMxTileRows = 128, kMxTileBlocks = 4, kMxTileBytes = 512;
constexpr uint32_t kScaleOne = 127u;            // the byte of 2^0; also that of a block without a finite value but zero

enum : int { TYPE_F32 = 0, TYPE_BF16 = 1, TYPE_F16 = 2 };

__host__ __device__ __forceinline__ int mx_blocks(int k) { return (k + kMxBlock - 1) / kMxBlock; }
__host__ __device__ __forceinline__ int mx_tiles_k(int k) { return (mx_blocks(k) + kMxTileBlocks - 1) / kMxTileBlocks; }
// Offset of the scale word of the four blocks 4 t .. 4 t + 3 of row r, in tiles.
__device__ __forceinline__ size_t mx_tile_word(size_t r, int t, int tiles_k) {
  return ((r >> 7) * static_cast<size_t>(tiles_k) + t) * kMxTileBytes + ((r & 31) << 4) + (((r >> 5) & 3) << 2);
}

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// Two values packed in a word of a 16-bit type, the first one low.
__device__ __forceinline__ uint32_t pack_two(float a, float b, __nv_bfloat16) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack_two(float a, float b, __half) {
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float2 unpack_two(uint32_t w, __nv_bfloat16) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
__device__ __forceinline__ float2 unpack_two(uint32_t w, __half) {
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}

// The checked build's test of an access: whether `count` bytes from p on are the tensor's.  (Elsewhere the constant true.)
#define QC_AT(extent, p, count) QC_IN((extent).has(p, count) ? 0 : 1, 1)

constexpr uint32_t kInfBits = 0x7F800000u;

// max(m, |a|, |b|) in one instruction; NaN if any of them is.
__device__ __forceinline__ float max_abs(float m, float a, float b) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(m), "f"(a), "f"(b));
  return r;
}
// The larger of each two 16-bit numbers.
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// How rows of values may be reached: in units of so many bytes (a power of two from the type's size to 32).  From kLoadUnit
// on (loads) or kStoreUnit (stores) a lane moves its own values; below, neighbouring lanes take neighbouring units and
// exchange them through shared memory (group_load).  8192 rows of 4096, 4100, 4098, 4097 bf16 take 16.5, 25.3, 29.0, 33.8 us to
// quantise.  Units of 16 bytes, own and exchanged: 8192 x 4100 float32 quantised in 28.9 and 39.1 us, read back in 41.8 and
// 35.9; 65536 x 72 bf16 6.3 and 6.2, back 8.9 and 5.6 (two stores a lane, each of parts of sectors).
constexpr int kLoadUnit = 16, kStoreUnit = 32;

// What a lane holds of a row: 32 bytes, E consecutive values (8 float32, 16 of a 16-bit type).
template <typename T> struct Piece {
  static constexpr int E = 32 / static_cast<int>(sizeof(T));
  uint32_t w[8];

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = 0u;
  }
  // Whole pieces.  (Ordinary loads, not the read-only path: the memory may be written by this kernel, too.)
  __device__ __forceinline__ void load(const T* p, int unit) {
    if (unit == 32) {
      asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                   : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
    } else {
      const uint4 a = *reinterpret_cast<const uint4*>(p), b = *(reinterpret_cast<const uint4*>(p) + 1);
      w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
    }
  }
  __device__ __forceinline__ void store(T* p, int unit) const {
    if (unit == 32) {
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                   ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
    } else {
      reinterpret_cast<uint4*>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
      reinterpret_cast<uint4*>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
  }
  __device__ __forceinline__ void unpack(float (&v)[E]) const {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < E; ++i) v[i] = __uint_as_float(w[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 f = unpack_two(w[i], T());
        v[2 * i] = f.x; v[2 * i + 1] = f.y;
      }
    }
  }
  __device__ __forceinline__ void pack(const float (&v)[E]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < E; ++i) w[i] = __float_as_uint(v[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = pack_two(v[2 * i], v[2 * i + 1], T());
    }
  }
  // Bits, as float32's, of the largest magnitude, at least infinity's if one is not finite; for 16-bit types two at a time
  // (magnitudes order like their bit patterns, NaN above infinity).
  __device__ __forceinline__ uint32_t top() const {
    if constexpr (sizeof(T) == 4) {
      float m = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; i += 2) m = max_abs(m, __uint_as_float(w[i]), __uint_as_float(w[i + 1]));
      return __float_as_uint(m);
    } else {
      uint32_t m = w[0] & 0x7FFF7FFFu;
#pragma unroll
      for (int i = 1; i < 8; ++i) m = max_u16x2(m, w[i] & 0x7FFF7FFFu);
      m = max(m & 0xFFFFu, m >> 16);
      if constexpr (static_cast<bool>(__is_same(T, __half)))
        return __float_as_uint(__half2float(__ushort_as_half(static_cast<unsigned short>(m))));
      else
        return m << 16;
    }
  }
};

// Bytes from or to p, which may be anywhere, for a group of G lanes (at least four): the first n of G * E.  Neighbouring
// lanes take neighbouring aligned words, and a few of them the bytes before the first and behind the last word.
struct ByteRun {
  int head, words, tail;
  __device__ __forceinline__ ByteRun(const void* p, int n) {
    n = max(n, 0);
    head = min(n, static_cast<int>(-reinterpret_cast<uintptr_t>(p) & 3));
    words = (n - head) >> 2;
    tail = (n - head) & 3;
  }
};
// From `bytes`, shared memory (4-byte aligned, readable up to the word behind the last byte's).
template <int E>
__device__ __forceinline__ void store_bytes(void* to, const uint8_t* bytes, int n, int G, int lane, const Extent& in) {
  const ByteRun run(to, n);
  uint8_t* p = static_cast<uint8_t*>(to);
  const uint32_t* words = reinterpret_cast<const uint32_t*>(bytes);
  if (lane < run.head && QC_AT(in, p + lane, 1)) p[lane] = bytes[lane];
#pragma unroll
  for (int i = 0; i < E / 4; ++i) {
    const int k = i * G + lane;
    if (k < run.words && QC_AT(in, p + run.head + 4 * k, 4))
      *reinterpret_cast<uint32_t*>(p + run.head + 4 * k) = __funnelshift_r(words[k], words[k + 1], 8 * run.head);
  }
  const int end = run.head + 4 * run.words + lane;
  if (lane < run.tail && QC_AT(in, p + end, 1)) p[end] = bytes[end];
}
// As loaded: a lane's words, and its byte before the first (low) and behind the last.  Then, through the group's part of the
// warp's shared memory, each lane's own E bytes; where there are none, anything.  Whole warps.
template <int E> struct DealtBytes {
  uint32_t w[E / 4], ends;
};
template <int E>
__device__ __forceinline__ void load_bytes(DealtBytes<E>& x, const void* from, int n, int G, int lane, const Extent& in) {
  const ByteRun run(from, n);
  const uint8_t* p = static_cast<const uint8_t*>(from);
#pragma unroll
  for (int i = 0; i < E / 4; ++i)
    x.w[i] = i * G + lane < run.words && QC_AT(in, p + run.head + 4 * (i * G + lane), 4)
                 ? *(reinterpret_cast<const uint32_t*>(p + run.head) + i * G + lane) : 0u;
  x.ends = lane < run.head && QC_AT(in, p + lane, 1) ? p[lane] : 0u;
  if (lane < run.tail && QC_AT(in, p + run.head + 4 * run.words + lane, 1)) x.ends |= static_cast<uint32_t>(p[run.head + 4 * run.words + lane]) << 8;
}
template <int E>
__device__ __forceinline__ void gather_bytes(uint32_t (&w)[E / 4], const DealtBytes<E>& x, const void* from, int n, int G, int lane, uint8_t* stage) {
  const ByteRun run(from, n);
  // byte b at `shift` + b: words stay words, and a lane's bytes begin in its first
  const int shift = -run.head & 3;
  uint8_t* group = stage + ((threadIdx.x & 31) - lane) * (E + 4);
  if (lane < run.head) group[shift + lane] = static_cast<uint8_t>(x.ends);
#pragma unroll
  for (int i = 0; i < E / 4; ++i)
    if (i * G + lane < run.words) reinterpret_cast<uint32_t*>(group + shift + run.head)[i * G + lane] = x.w[i];
  if (lane < run.tail) group[shift + run.head + 4 * run.words + lane] = static_cast<uint8_t>(x.ends >> 8);
  __syncwarp();
  const uint8_t* q = group + lane * E;
  uint32_t v[E / 4 + 1];
  if constexpr (E == 8) {
    const uint2 a = *reinterpret_cast<const uint2*>(q);
    v[0] = a.x; v[1] = a.y;
  } else {
#pragma unroll
    for (int i = 0; i < E / 16; ++i) {
      const uint4 a = reinterpret_cast<const uint4*>(q)[i];
      v[4 * i] = a.x; v[4 * i + 1] = a.y; v[4 * i + 2] = a.z; v[4 * i + 3] = a.w;
    }
  }
  v[E / 4] = *reinterpret_cast<const uint32_t*>(q + E);
#pragma unroll
  for (int i = 0; i < E / 4; ++i) w[i] = __funnelshift_r(v[i], v[i + 1], 8 * shift);
  __syncwarp();
}

// Bytes of shared memory a warp needs to exchange values: 36 a lane (gather_bytes).
constexpr int kWarpStage = 1152;

// The bits of a unit of U bytes.
template <int U> struct UnitOf { using type = uint32_t; };
template <> struct UnitOf<8> { using type = uint2; };
template <> struct UnitOf<16> { using type = uint4; };

// Unit i of a piece that holds units lane, lane + G, lane + 2 G, ... of a group's values (dealt pieces).
template <int U> __device__ __forceinline__ typename UnitOf<U>::type unit_of(const uint32_t (&w)[8], int i) {
  if constexpr (U == 16) return make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
  else if constexpr (U == 8) return make_uint2(w[2 * i], w[2 * i + 1]);
  else return w[i];
}
template <int U> __device__ __forceinline__ void set_unit(uint32_t (&w)[8], int i, typename UnitOf<U>::type v) {
  if constexpr (U == 16) { w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w; }
  else if constexpr (U == 8) { w[2 * i] = v.x; w[2 * i + 1] = v.y; }
  else w[i] = v;
}

// Dealt pieces from p, where n values exist (zeros behind them), and back; units of U bytes.
template <int U, typename T>
__device__ __forceinline__ void load_dealt(Piece<T>& x, const T* p, int n, int G, int lane, const Extent& in) {
  using Unit = typename UnitOf<U>::type;
  constexpr int kValues = U / static_cast<int>(sizeof(T));   // of a unit
#pragma unroll
  for (int i = 0; i < 32 / U; ++i) {
    const int at = (i * G + lane) * kValues, left = n - at;
    Unit v{};
    if (left >= kValues) {
      if (QC_AT(in, p + at, U)) v = *reinterpret_cast<const Unit*>(p + at);
    } else if (kValues > 1 && left > 0 && QC_AT(in, p + at, left * sizeof(T))) {   // (the row ends inside a unit)
      T part[kValues];
#pragma unroll
      for (int k = 0; k < kValues; ++k) part[k] = k < left ? p[at + k] : from_float<T>(0.0f);
      memcpy(&v, part, U);
    }
    set_unit<U>(x.w, i, v);
  }
}
template <int U, typename T>
__device__ __forceinline__ void store_dealt(const Piece<T>& x, T* p, int n, int G, int lane, const Extent& in) {
  using Unit = typename UnitOf<U>::type;
  constexpr int kValues = U / static_cast<int>(sizeof(T));
#pragma unroll
  for (int i = 0; i < 32 / U; ++i) {
    const int at = (i * G + lane) * kValues, left = n - at;
    const Unit v = unit_of<U>(x.w, i);
    if (left >= kValues) {
      if (QC_AT(in, p + at, U)) *reinterpret_cast<Unit*>(p + at) = v;
    } else if (kValues > 1 && left > 0 && QC_AT(in, p + at, left * sizeof(T))) {
      T part[kValues];
      memcpy(part, &v, U);
#pragma unroll
      for (int k = 0; k < kValues; ++k)
        if (k < left) p[at + k] = part[k];
    }
  }
}
// Dealt pieces to those of consecutive values and back, through the warp's shared memory.  Whole warps.
template <int U, typename T>
__device__ __forceinline__ void gather_dealt(Piece<T>& x, int G, int lane, uint8_t* stage) {
  using Unit = typename UnitOf<U>::type;
  uint8_t* group = stage + ((threadIdx.x & 31) - lane) * 32;
#pragma unroll
  for (int i = 0; i < 32 / U; ++i) reinterpret_cast<Unit*>(group)[i * G + lane] = unit_of<U>(x.w, i);
  __syncwarp();
  const uint4* q = reinterpret_cast<const uint4*>(group + lane * 32);
  const uint4 a = q[0], b = q[1];
  x.w[0] = a.x; x.w[1] = a.y; x.w[2] = a.z; x.w[3] = a.w; x.w[4] = b.x; x.w[5] = b.y; x.w[6] = b.z; x.w[7] = b.w;
  __syncwarp();
}
template <int U, typename T>
__device__ __forceinline__ void deal(Piece<T>& x, int G, int lane, uint8_t* stage) {
  using Unit = typename UnitOf<U>::type;
  uint8_t* group = stage + ((threadIdx.x & 31) - lane) * 32;
  uint4* q = reinterpret_cast<uint4*>(group + lane * 32);
  q[0] = make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]);
  q[1] = make_uint4(x.w[4], x.w[5], x.w[6], x.w[7]);
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 32 / U; ++i) set_unit<U>(x.w, i, reinterpret_cast<const Unit*>(group)[i * G + lane]);
  __syncwarp();
}
// f(the unit as a constant, 4 to 16 bytes) for a unit that is the same for the whole grid.
template <typename F> __device__ __forceinline__ void with_unit(int unit, F&& f) {
  if (unit >= 16) f(std::integral_constant<int, 16>());
  else if (unit == 8) f(std::integral_constant<int, 8>());
  else f(std::integral_constant<int, 4>());
}
// Rows of a 16-bit type that reach 2 bytes alone: by words and, at the ends, bytes; the gathered piece has zeros behind the n
// values.
template <typename T> __device__ __forceinline__ bool by_bytes(int unit) { return sizeof(T) == 2 && unit == 2; }
template <typename T>
__device__ __forceinline__ int byte_count(int n, int G) { return min(n, G * Piece<T>::E) * static_cast<int>(sizeof(T)); }
template <typename T>
__device__ __forceinline__ void load_piece(Piece<T>& x, uint32_t& ends, const T* p, int n, int G, int lane, const Extent& in) {
  DealtBytes<32> dealt;
  load_bytes<32>(dealt, p, byte_count<T>(n, G), G, lane, in);
#pragma unroll
  for (int i = 0; i < 8; ++i) x.w[i] = dealt.w[i];
  ends = dealt.ends;
}
template <typename T>
__device__ __forceinline__ void gather_piece(Piece<T>& x, uint32_t ends, const T* p, int n, int G, int lane, uint8_t* stage) {
  DealtBytes<32> dealt;
#pragma unroll
  for (int i = 0; i < 8; ++i) dealt.w[i] = x.w[i];
  dealt.ends = ends;
  gather_bytes<32>(x.w, dealt, p, byte_count<T>(n, G), G, lane, stage);
  const int left = n - lane * Piece<T>::E;
  if (left < Piece<T>::E)
#pragma unroll
    for (int i = 0; i < 8; ++i) x.w[i] = left >= 2 * i + 2 ? x.w[i] : left == 2 * i + 1 ? x.w[i] & 0xFFFFu : 0u;
}
template <typename T>
__device__ __forceinline__ void store_piece(const Piece<T>& x, T* p, int n, int G, int lane, uint8_t* stage, const Extent& in) {
  uint8_t* group = stage + ((threadIdx.x & 31) - lane) * 32;
  uint4* q = reinterpret_cast<uint4*>(group + lane * 32);
  q[0] = make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]);
  q[1] = make_uint4(x.w[4], x.w[5], x.w[6], x.w[7]);
  __syncwarp();
  store_bytes<32>(p, group, byte_count<T>(n, G), G, lane, in);
  __syncwarp();
}

// Loads the pieces of a group of G lanes (a power of two up to 32): G * E consecutive values from p on, of which the first
// n exist (zeros behind them; n may be negative).  ANY: exchanged (an instantiation of its own, so that the
// aligned one is lean).  Whole warps.
template <bool ANY, typename T>
__device__ __forceinline__ void group_load(Piece<T>& x, const T* p, int n, int G, int lane, int unit, uint8_t* stage, const Extent& in) {
  constexpr int E = Piece<T>::E;
  if constexpr (!ANY) {
    const int left = n - lane * E;
    const bool here = left > 0 && QC_AT(in, p + lane * E, min(left, E) * sizeof(T));
    if (left >= E && here) {
      x.load(p + lane * E, unit);
    } else {
      x.clear();
      constexpr int kValues = 4 / static_cast<int>(sizeof(T));
      if (here) {                                        // the row's end, in words
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (left >= (i + 1) * kValues) x.w[i] = reinterpret_cast<const uint32_t*>(p + lane * E)[i];
          else if (kValues == 2 && left == 2 * i + 1) x.w[i] = reinterpret_cast<const unsigned short*>(p + lane * E)[2 * i];
        }
      }
    }
  } else {
    if (by_bytes<T>(unit)) {
      uint32_t ends;
      load_piece(x, ends, p, n, G, lane, in);
      gather_piece(x, ends, p, n, G, lane, stage);
    } else {
      with_unit(unit, [&](auto u) {
        load_dealt<decltype(u)::value>(x, p, n, G, lane, in);
        gather_dealt<decltype(u)::value>(x, G, lane, stage);
      });
    }
  }
}
// The same way back: the first n values.
template <bool ANY, typename T>
__device__ __forceinline__ void group_store(const Piece<T>& x, T* p, int n, int G, int lane, int unit, uint8_t* stage, const Extent& in) {
  constexpr int E = Piece<T>::E;
  if constexpr (!ANY) {
    const int left = n - lane * E;
    const bool here = left > 0 && QC_AT(in, p + lane * E, min(left, E) * sizeof(T));
    if (left >= E && here) {
      x.store(p + lane * E, unit);
    } else if (here) {
      constexpr int kValues = 4 / static_cast<int>(sizeof(T));
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (left >= (i + 1) * kValues) reinterpret_cast<uint32_t*>(p + lane * E)[i] = x.w[i];
        else if (kValues == 2 && left == 2 * i + 1) reinterpret_cast<unsigned short*>(p + lane * E)[2 * i] = static_cast<unsigned short>(x.w[i]);
      }
    }
  } else {
    if (by_bytes<T>(unit)) {
      store_piece(x, p, n, G, lane, stage, in);
    } else {
      with_unit(unit, [&](auto u) {
        Piece<T> dealt = x;
        deal<decltype(u)::value>(dealt, G, lane, stage);
        store_dealt<decltype(u)::value>(dealt, p, n, G, lane, in);
      });
    }
  }
}

// Bits of the largest |v| over a lane's values, at least infinity's if one is not finite; over the finite ones alone, with
// NaN made 0 in v (infinities stay: they saturate).
template <int E>
__device__ __forceinline__ uint32_t top_bits(const float (&v)[E]) {
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < E; i += 2) m = max_abs(m, v[i], v[i + 1]);
  return __float_as_uint(m);
}
template <int E>
__device__ __forceinline__ uint32_t top_bits_finite(float (&v)[E]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const uint32_t a = __float_as_uint(v[i]) & 0x7FFFFFFFu;
    if (a > kInfBits) v[i] = 0.0f;
    else if (a < kInfBits) m = max(m, a);
  }
  return m;
}
template <int LANES>
__device__ __forceinline__ uint32_t max_over(uint32_t m) {
#pragma unroll
  for (int d = 1; d < LANES; d *= 2) m = max(m, __shfl_xor_sync(0xffffffffu, m, d));
  return m;
}
// Largest finite magnitude of the values that LANES neighbouring lanes hold; NaN becomes 0 in v.  m: top_bits of v, if that is
// known already.  Whole warps only.
template <int LANES, int E>
__device__ __forceinline__ uint32_t finite_top(float (&v)[E], uint32_t m) {
  if (__any_sync(0xffffffffu, m >= kInfBits)) m = top_bits_finite(v);
  return max_over<LANES>(m);
}

// Scale byte of a block of 4-bit values whose largest finite magnitude has the bits m (0: the block is zero, scale 1).
// round_up = 0x3FFFFF: the smallest e with 6 * 2^e >= top, i.e. e + 127 = exponent field - 2, one more when the significand
// is above 1.5 (the addition carries).  round_up = 0: e = floor(log2 top) - 2, with values above 6 * 2^e saturating.
constexpr uint32_t kCoverRoundUp = 0x3FFFFFu;
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t m, uint32_t round_up) {
  const int s = static_cast<int>((m + round_up) >> 23) - 2;
  return m == 0u ? kScaleOne : static_cast<uint32_t>(max(s, 0));
}
// Scale byte of int8 values: the smallest e >= -126 with 127 * 2^e >= top (127 = 1.984375 * 2^6).
__device__ __forceinline__ uint32_t i8_scale_byte(uint32_t m) {
  const int s = static_cast<int>((m + 0x1FFFFu) >> 23) - 6;
  return m == 0u ? kScaleOne : static_cast<uint32_t>(max(s, 1));
}
// 2^-e of a scale byte up to 253 (what the two functions above give).
__device__ __forceinline__ float inverse_scale(uint32_t s) { return __uint_as_float((254u - s) << 23); }
// 2^e of any scale byte; 255 stands for NaN.
__device__ __forceinline__ float scale_of(uint32_t s) {
  return __uint_as_float(s == 0u ? 0x00400000u : s == 255u ? 0x7FC00000u : s << 23);
}

// Eight values, scaled, to eight codes, the first in the low four bits: nearest, ties to the even pattern, saturating (the
// conversion instruction's own rule), and a zero magnitude always code 0 (it leaves the sign on small negative values).
__device__ __forceinline__ uint32_t mx_encode_eight(const float* v, float inv) {
  uint32_t w;
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
      "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
      : "=r"(w)
      : "f"(v[0] * inv), "f"(v[1] * inv), "f"(v[2] * inv), "f"(v[3] * inv), "f"(v[4] * inv), "f"(v[5] * inv), "f"(v[6] * inv),
        "f"(v[7] * inv));
  const uint32_t mag = w & 0x77777777u;
  return mag | (w & (mag + 0x77777777u) & 0x88888888u);      // a magnitude from 1 to 7 carries into bit 3
}
__device__ __forceinline__ void mx_decode_eight(uint32_t w, float scale, float* v) {
  uint32_t h[4];
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
      "mov.b32 {b0, b1, b2, b3}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, b0;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, b2;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(w));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = unpack_two(h[i], __half());
    v[2 * i] = f.x * scale; v[2 * i + 1] = f.y * scale;
  }
}

// Four values, scaled, to int8 codes in +-127: nearest even, NaN to 0 (the conversion's rule, kept alive by the maximum that
// hands NaN on), saturated as they are packed.
__device__ __forceinline__ uint32_t i8_encode_four(const float* v, float inv) {
  int c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float t;
    asm("max.NaN.f32 %0, %1, 0fC2FE0000;" : "=f"(t) : "f"(v[i] * inv));          // -127
    c[i] = __float2int_rn(t);
  }
  uint32_t lo, all;
  asm("cvt.pack.sat.s8.s32.b32 %0, %1, %2, 0;" : "=r"(lo) : "r"(c[3]), "r"(c[2]));
  asm("cvt.pack.sat.s8.s32.b32 %0, %1, %2, %3;" : "=r"(all) : "r"(c[1]), "r"(c[0]), "r"(lo));
  return all;
}
// Four int8 codes to values: a byte with its sign bit turned is the low byte of the float 2^23 + 128 + code.
__device__ __forceinline__ void i8_decode_four(uint32_t w, float scale, float* v) {
  const uint32_t b = w ^ 0x80808080u;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = (__uint_as_float(__byte_perm(b, 0x4B000000u, 0x7440 + i)) - 8388736.0f) * scale;
}

// Codes of a lane's E values in 4 bits.
template <int E>
__device__ __forceinline__ void mx_store_codes(uint8_t* p, const float (&v)[E], float inv, const Extent& in) {
  if (!QC_AT(in, p, E / 2)) return;
  if constexpr (E == 8) *reinterpret_cast<uint32_t*>(p) = mx_encode_eight(v, inv);
  else *reinterpret_cast<uint2*>(p) = make_uint2(mx_encode_eight(v, inv), mx_encode_eight(v + 8, inv));
}

// Where a row's scales go.
struct MxScales {
  uint8_t* bytes;
  int tiles;            // 1: in tiles, 0: row by row
  int blocks, tiles_k;
  size_t extent;        // bytes of the whole array
};
// The word of blocks 4 t .. 4 t + 3 of row r, in tiles (with the bytes behind the row's last block: a byte of 2^0 each).
__device__ __forceinline__ void store_scale_word(const MxScales& s, size_t r, int t, uint32_t word) {
  const size_t at = mx_tile_word(r, t, s.tiles_k);
  if (QC_AT(Extent::of(s.bytes, s.extent), s.bytes + at, 4)) *reinterpret_cast<uint32_t*>(s.bytes + at) = word;
}
// The scale byte s of the block of which this lane's values, from column `col` of row r on, are a part.  Every lane of a warp
// calls it (`here`: the lane has values or their padding); LANES lanes a block.
template <int LANES>
__device__ __forceinline__ void store_scale(const MxScales& scales, size_t r, int col, uint32_t s, bool here) {
  if (scales.tiles) {
    // four blocks at once
    s |= __shfl_down_sync(0xffffffffu, s, LANES) << 8;
    s |= __shfl_down_sync(0xffffffffu, s, 2 * LANES) << 16;
    if (here && (col & 127) == 0) store_scale_word(scales, r, col >> 7, s);
  } else if (here && (col & (kMxBlock - 1)) == 0) {
    const size_t at = r * static_cast<size_t>(scales.blocks) + col / kMxBlock;
    if (QC_IN(at, scales.extent)) scales.bytes[at] = static_cast<uint8_t>(s);
  }
}

}  // namespace qc
