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
template <int TYPE> struct TypeOf { using type = float; };
template <> struct TypeOf<TYPE_BF16> { using type = __nv_bfloat16; };
template <> struct TypeOf<TYPE_F16> { using type = __half; };

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

// Eight consecutive values of a row, as they lie in memory (16 or 32 bytes).
template <typename T> struct Eight {
  uint4 w[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T)) / 2; ++i) w[i] = __ldg(reinterpret_cast<const uint4*>(p) + i);
  }
  // The same through the ordinary path, for memory that this kernel also writes.
  __device__ __forceinline__ void load_written(const T* p) {
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T)) / 2; ++i) w[i] = reinterpret_cast<const uint4*>(p)[i];
  }
  __device__ __forceinline__ void unpack(float (&v)[8]) const {
    if constexpr (sizeof(T) == 4) {
      v[0] = __uint_as_float(w[0].x); v[1] = __uint_as_float(w[0].y); v[2] = __uint_as_float(w[0].z); v[3] = __uint_as_float(w[0].w);
      v[4] = __uint_as_float(w[1].x); v[5] = __uint_as_float(w[1].y); v[6] = __uint_as_float(w[1].z); v[7] = __uint_as_float(w[1].w);
    } else {
      const uint32_t q[4] = {w[0].x, w[0].y, w[0].z, w[0].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 f = unpack_two(q[i], T());
        v[2 * i] = f.x; v[2 * i + 1] = f.y;
      }
    }
  }
  __device__ __forceinline__ void pack(const float (&v)[8]) {
    if constexpr (sizeof(T) == 4) {
      w[0] = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
      w[1] = make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
    } else {
      w[0] = make_uint4(pack_two(v[0], v[1], T()), pack_two(v[2], v[3], T()), pack_two(v[4], v[5], T()), pack_two(v[6], v[7], T()));
    }
  }
  __device__ __forceinline__ void store(T* p) const {
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T)) / 2; ++i) reinterpret_cast<uint4*>(p)[i] = w[i];
  }
};

// The first `n` of eight values at p one by one, zeros behind them.
template <typename T>
__device__ __forceinline__ void load_some(const T* p, int n, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = i < n ? to_float(p[i]) : 0.0f;
}
template <typename T>
__device__ __forceinline__ void store_some(T* p, int n, const float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) p[i] = from_float<T>(v[i]);
}

constexpr uint32_t kInfBits = 0x7F800000u;

// Bits of the largest |v| (magnitudes order like their bit patterns, NaN above infinity).
__device__ __forceinline__ uint32_t top_bits(const float (&v)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
  return m;
}
// The same over the finite values alone; NaN becomes 0 in v, infinities stay (they saturate).
__device__ __forceinline__ uint32_t top_bits_finite(float (&v)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
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
// Largest finite magnitude of the 8 LANES values that LANES neighbouring lanes hold; NaN becomes 0 in v.  Whole warps only.
template <int LANES>
__device__ __forceinline__ uint32_t finite_top(float (&v)[8]) {
  uint32_t m = top_bits(v);
  if (__any_sync(0xffffffffu, m >= kInfBits)) m = top_bits_finite(v);
  return max_over<LANES>(m);
}

// Scale byte of a block of 4-bit values whose largest finite magnitude has the bits m (0: the block is zero, scale 1).
// round_up = 0x3FFFFF: the smallest e with 6 * 2^e >= top, i.e. e + 127 = exponent field - 2, one more when the significand
// is above 1.5 (the addition carries).  round_up = 0: e = floor(log2 top) - 2, with values above 6 * 2^e saturating.
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

// Eight scaled values to eight codes, the first in the low four bits: nearest, ties to the even pattern, saturating (the
// conversion instruction's own rule), and a zero magnitude always code 0 (it leaves the sign on small negative values).
__device__ __forceinline__ uint32_t mx_encode_eight(const float (&v)[8], float inv) {
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
__device__ __forceinline__ void mx_decode_eight(uint32_t w, float scale, float (&v)[8]) {
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

// Eight scaled values to int8 codes in +-127, nearest even, NaN to 0: {codes 0-3, codes 4-7}.
__device__ __forceinline__ uint2 i8_encode_eight(const float (&v)[8], float inv) {
  uint32_t c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float t = fminf(fmaxf(v[i] * inv, -127.0f), 127.0f);
    c[i] = static_cast<uint32_t>(v[i] == v[i] ? __float2int_rn(t) : 0) & 0xFFu;
  }
  return make_uint2(c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24, c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24);
}
__device__ __forceinline__ void i8_decode_eight(uint2 w, float scale, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = static_cast<float>(static_cast<int8_t>(w.x >> (8 * i))) * scale;
    v[4 + i] = static_cast<float>(static_cast<int8_t>(w.y >> (8 * i))) * scale;
  }
}

// The scale bytes of four consecutive blocks, one held by every fourth lane of sixteen, as one word (valid in the first
// of the sixteen lanes).
__device__ __forceinline__ uint32_t gather_scale_word(uint32_t s) {
  s |= __shfl_down_sync(0xffffffffu, s, 4) << 8;
  return s | __shfl_down_sync(0xffffffffu, s, 8) << 16;
}

// Where a row's scales go.
struct MxScales {
  uint8_t* bytes;
  int tiles;            // 1: in tiles, 0: row by row
  int blocks, tiles_k;
  size_t extent;        // bytes of the whole array
};
// The word of blocks 4 t .. 4 t + 3 of row r; in tiles also the bytes behind the row's last block (a byte of 2^0 each).
__device__ __forceinline__ void store_scale_word(const MxScales& s, size_t r, int t, uint32_t word) {
  if (s.tiles) {
    const size_t at = mx_tile_word(r, t, s.tiles_k);
    if (QC_IN(at + 3, s.extent)) *reinterpret_cast<uint32_t*>(s.bytes + at) = word;
  } else {
    const size_t at = r * static_cast<size_t>(s.blocks) + 4 * t;
    const int n = min(4, s.blocks - 4 * t);
    if (!QC_IN(at + n - 1, s.extent)) return;
    if (n == 4 && (reinterpret_cast<uintptr_t>(s.bytes + at) & 3) == 0) *reinterpret_cast<uint32_t*>(s.bytes + at) = word;
    else
      for (int i = 0; i < n; ++i) s.bytes[at + i] = static_cast<uint8_t>(word >> (8 * i));
  }
}

}  // namespace qc
