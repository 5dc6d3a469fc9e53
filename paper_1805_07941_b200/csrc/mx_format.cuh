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

#include "epilogue.cuh"

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

// How a row of values may be reached.
enum : int { ROWS_ANY = 0, ROWS_16 = 1, ROWS_32 = 2 };     // one value at a time; in 16-byte pieces; in 32-byte pieces

// What a lane holds of a row: 32 bytes, E consecutive values (8 float32, 16 of a 16-bit type).
template <typename T> struct Piece {
  static constexpr int E = 32 / static_cast<int>(sizeof(T));
  uint32_t w[8];

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = 0u;
  }
  // Whole pieces.  (Ordinary loads, not the read-only path: the memory may be written by this kernel, too.)
  __device__ __forceinline__ void load(const T* p, int how) {
    if (how == ROWS_32) {
      asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                   : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
    } else {
      const uint4 a = *reinterpret_cast<const uint4*>(p), b = *(reinterpret_cast<const uint4*>(p) + 1);
      w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
    }
  }
  __device__ __forceinline__ void store(T* p, int how) const {
    if (how == ROWS_32) {
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

// Bytes of shared memory a warp needs for rows that are reached one value at a time.
constexpr int kWarpStage = 1024;

// Lane l of a group of G holds values l, l + G, l + 2 G, ... and gets E consecutive ones, through its warp's shared memory.
template <typename T>
__device__ __forceinline__ void group_arrange(Piece<T>& x, const T (&v)[Piece<T>::E], int G, int lane, uint8_t* stage) {
  constexpr int E = Piece<T>::E;
  T* mine = reinterpret_cast<T*>(stage) + ((threadIdx.x & 31) - lane) * E;
#pragma unroll
  for (int i = 0; i < E; ++i) mine[i * G + lane] = v[i];
  __syncwarp();
  const uint4* q = reinterpret_cast<const uint4*>(mine + lane * E);
  const uint4 a = q[0], b = q[1];
  x.w[0] = a.x; x.w[1] = a.y; x.w[2] = a.z; x.w[3] = a.w; x.w[4] = b.x; x.w[5] = b.y; x.w[6] = b.z; x.w[7] = b.w;
  __syncwarp();
}

// Loads the pieces of a group of G lanes (a power of two up to 32): G * E consecutive values from p on, of which the first
// n exist (zeros behind them; n may be negative).  Where 16-byte accesses are not aligned the group reads one value a
// lane, neighbouring lanes neighbouring values, and passes them through its warp's shared memory.  Whole warps.  ANY: how is
// ROWS_ANY (an instantiation of its own, so that the aligned one is lean).
template <bool ANY, typename T>
__device__ __forceinline__ void group_load(Piece<T>& x, const T* p, int n, int G, int lane, int how, uint8_t* stage) {
  constexpr int E = Piece<T>::E;
  if constexpr (!ANY) {
    const int left = n - lane * E;
    if (left >= E) {
      x.load(p + lane * E, how);
    } else {
      x.clear();
      if (left > 0) {
        float v[E];
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = i < left ? to_float(p[lane * E + i]) : 0.0f;
        x.pack(v);
      }
    }
  } else {
    T v[E];
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = i * G + lane < n ? p[i * G + lane] : from_float<T>(0.0f);
    group_arrange(x, v, G, lane, stage);
  }
}
// The same way back: the first n values.
template <bool ANY, typename T>
__device__ __forceinline__ void group_store(const Piece<T>& x, T* p, int n, int G, int lane, int how, uint8_t* stage) {
  constexpr int E = Piece<T>::E;
  if constexpr (!ANY) {
    const int left = n - lane * E;
    if (left >= E) {
      x.store(p + lane * E, how);
    } else if (left > 0) {
      float v[E];
      x.unpack(v);
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (i < left) p[lane * E + i] = from_float<T>(v[i]);
    }
  } else {
    T* mine = reinterpret_cast<T*>(stage) + ((threadIdx.x & 31) - lane) * E;
    uint4* q = reinterpret_cast<uint4*>(mine + lane * E);
    q[0] = make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]);
    q[1] = make_uint4(x.w[4], x.w[5], x.w[6], x.w[7]);
    __syncwarp();
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (i * G + lane < n) p[i * G + lane] = mine[i * G + lane];
    __syncwarp();
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
__device__ __forceinline__ void mx_store_codes(uint8_t* p, const float (&v)[E], float inv) {
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
  if (QC_IN(at + 3, s.extent)) *reinterpret_cast<uint32_t*>(s.bytes + at) = word;
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
