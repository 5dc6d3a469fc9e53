// Tensors to microscaled 4-bit codes and back (mx_format.cuh has the type).  Both directions are bound by HBM: 2 or 4
// bytes in and 17/32 out per value, or the other way round.  Sixteen lanes take 128 consecutive values of a row, eight
// each (16-byte accesses): a block is four lanes, its maximum two shuffles, and the four scales of the sixteen lanes are one word.
#pragma once
#include "mx_format.cuh"
#include "kernel_igemm.cuh"

namespace qc {

constexpr int kMxThreads = 256;
constexpr int kMxUnroll = 4;                    // pieces of 128 values a half-warp has in flight

// Units: 128-value piece g of row r, r slowest.  In tiles the rows up to the next multiple of 128 have units too, which
// write their scale words (2^0) alone.
template <typename T>
__global__ void __launch_bounds__(kMxThreads)
mx_quantize_kernel(const T* __restrict__ x, size_t ld, size_t rows, int K, uint8_t* __restrict__ codes, MxScales scales, uint32_t round_up,
                   int units, FastDiv fd_pieces, int vec_ok) {
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const int lane16 = threadIdx.x & 15;
  const int halves = gridDim.x * (kMxThreads / 16);
  const size_t code_pitch = static_cast<size_t>(scales.blocks) * 16;
  // both halves of a warp run the same number of rounds
  const int first = blockIdx.x * (kMxThreads / 16) + (threadIdx.x >> 4), first_even = first & ~1;
  for (int base = first_even; base < units; base += halves * kMxUnroll) {
    float v[kMxUnroll][8];
#pragma unroll
    for (int j = 0; j < kMxUnroll; ++j) {
      const int u = base + (first & 1) + j * halves;
      int g = 0;
      const size_t r = u < units ? fd_pieces.divmod(u, &g) : rows;
      const int col = g * 128 + lane16 * 8, n = K - col;
      const T* p = x + r * ld + col;
      if (r < rows && n >= 8 && vec_ok && QC_IN(r * ld + col + 7, (rows - 1) * ld + K)) {
        Eight<T> e;
        e.load(p);
        e.unpack(v[j]);
      } else if (r < rows && n > 0 && QC_IN(r * ld + col + min(n, 8) - 1, (rows - 1) * ld + K)) {
        load_some(p, n, v[j]);
      } else {
        load_some(p, 0, v[j]);
      }
    }
#pragma unroll
    for (int j = 0; j < kMxUnroll; ++j) {
      const int u = base + (first & 1) + j * halves;
      if (base + j * halves >= units) break;                // (the same for the whole warp: base is even)
      int g = 0;
      const size_t r = u < units ? fd_pieces.divmod(u, &g) : rows;
      const uint32_t s = mx_scale_byte(finite_top<4>(v[j]), round_up);
      const uint32_t word = gather_scale_word(s);
      const int at = g * 64 + lane16 * 4;                   // byte of the row's codes
      if (r < rows && at < scales.blocks * 16 && QC_IN(r * code_pitch + at + 3, rows * code_pitch))
        *reinterpret_cast<uint32_t*>(codes + r * code_pitch + at) = mx_encode_eight(v[j], inverse_scale(s));
      if (lane16 == 0 && u < units) store_scale_word(scales, r, g, word);
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kMxThreads)
mx_dequantize_kernel(const uint8_t* __restrict__ codes, MxScales scales, size_t rows, int K, T* __restrict__ y, size_t ld, int units,
                     FastDiv fd_pieces, int vec_ok) {
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const int lane16 = threadIdx.x & 15;
  const int halves = gridDim.x * (kMxThreads / 16);
  const size_t code_pitch = static_cast<size_t>(scales.blocks) * 16;
  for (int base = blockIdx.x * (kMxThreads / 16) + (threadIdx.x >> 4); base < units; base += halves * kMxUnroll) {
    uint32_t w[kMxUnroll], s[kMxUnroll];
#pragma unroll
    for (int j = 0; j < kMxUnroll; ++j) {
      const int u = base + j * halves;
      w[j] = 0; s[j] = kScaleOne;
      if (u >= units) continue;
      int g;
      const size_t r = fd_pieces.divmod(u, &g);
      const int b = g * 4 + (lane16 >> 2);
      if (b >= scales.blocks) continue;
      const size_t at = r * code_pitch + g * 64 + lane16 * 4;
      const size_t sat = scales.tiles ? mx_tile_word(r, g, scales.tiles_k) + (b & 3) : r * static_cast<size_t>(scales.blocks) + b;
      if (!QC_IN(at + 3, rows * code_pitch) || !QC_IN(sat, scales.extent)) continue;
      w[j] = __ldg(reinterpret_cast<const uint32_t*>(codes + at));
      s[j] = __ldg(scales.bytes + sat);
    }
#pragma unroll
    for (int j = 0; j < kMxUnroll; ++j) {
      const int u = base + j * halves;
      if (u >= units) break;
      int g;
      const size_t r = fd_pieces.divmod(u, &g);
      const int col = g * 128 + lane16 * 8, n = K - col;
      if (n <= 0 || !QC_IN(r * ld + col + min(n, 8) - 1, (rows - 1) * ld + K)) continue;
      float v[8];
      mx_decode_eight(w[j], scale_of(s[j]), v);
      if (vec_ok && n >= 8) {
        Eight<T> e;
        e.pack(v);
        e.store(y + r * ld + col);
      } else {
        store_some(y + r * ld + col, n, v);
      }
    }
  }
}

}  // namespace qc
