// Tensors to microscaled 4-bit codes and back (mx_format.cuh has the type).  Both directions are bound by HBM: 2 or 4
// bytes in and 17/32 out per value, or the other way round.  A lane takes 32 bytes of values, so that a block is two or
// four lanes (its maximum one or two shuffles) and the scales of eight or sixteen lanes are one word.  A thread stays in its
// columns and walks down the rows, so that an address is one product and no division is left.  One row at a time and 48
// warps an SM; two rows at a time and 32 warps, or 24, were slower (8192 x 8192 bf16 33 us against 34 and 40).
// 8192 x 8192 bf16: quantised in 34 us (0.78 of the measured copy rate, 63 % of the issue slots), read back in 30 (0.88);
// 8192 x 5000 float32: 32 us each way (0.89).
#pragma once
#include "mx_format.cuh"
#include "kernel_igemm.cuh"

namespace qc {

constexpr int kMxThreads = 256;
// Blocks of an SM.  ANY: six leave 40 registers, which spill (8192 x 4098 bf16 quantised in 31.4 us, 30.0 with four; 65536 x 68
// 7.9 and 6.0).
template <bool ANY> constexpr int kMxBlocks = ANY ? 4 : 6;

// A block is lanes_x lanes (a power of two, at least those of a scale word) along the row by kMxThreads / lanes_x rows.
struct MxGrid {
  int lanes_x, log_x;
  size_t rows;            // of the tensor
  size_t rows_out;        // with the rows that fill up the last tile (quantisation into tiles)
  int K;
  size_t ld;
  int unit;               // bytes that rows of values may be reached in
};

template <typename T, bool ANY>
__global__ void __launch_bounds__(kMxThreads, kMxBlocks<ANY>)
mx_quantize_kernel(const T* __restrict__ x, const MxGrid g, uint8_t* __restrict__ codes, const MxScales scales, uint32_t round_up) {
  constexpr int E = Piece<T>::E, kBlockLanes = kMxBlock / E;
  __shared__ __align__(16) uint8_t stage[ANY ? kMxThreads / 32 : 1][ANY ? kWarpStage : 1];
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const int G = min(g.lanes_x, 32);
  const int lane_x = threadIdx.x & (g.lanes_x - 1), lane = lane_x & (G - 1);
  const int col = (static_cast<int>(blockIdx.x) * g.lanes_x + lane_x) * E, first = col - lane * E;   // of the lane, of its group
  const size_t pitch = static_cast<size_t>(scales.blocks) * 16;
  const size_t step = static_cast<size_t>(gridDim.y) * (kMxThreads >> g.log_x);
  const bool codes_here = col < scales.blocks * kMxBlock;
  uint8_t* my_stage = stage[ANY ? threadIdx.x >> 5 : 0];
  const Extent of_x = Extent::of(x, (g.rows - 1) * g.ld + g.K), of_codes = Extent::of(codes, g.rows * pitch);
  // every lane of a warp goes round as often as the warp's first
  const size_t warp_row = (threadIdx.x & ~31u) >> g.log_x, my_row = (threadIdx.x >> g.log_x) - warp_row;
  for (size_t base = blockIdx.y * static_cast<size_t>(kMxThreads >> g.log_x) + warp_row; base < g.rows_out; base += step) {
    const size_t r = base + my_row;
    Piece<T> p;
    group_load<ANY>(p, x + r * g.ld + first, r < g.rows ? g.K - first : 0, G, lane, g.unit, my_stage, of_x);
    float v[E];
    p.unpack(v);
    const uint32_t s = mx_scale_byte(finite_top<kBlockLanes>(v, p.top()), round_up);
    if (codes_here && r < g.rows) mx_store_codes(codes + r * pitch + col / 2, v, inverse_scale(s), of_codes);
    store_scale<kBlockLanes>(scales, r, col, s, codes_here && r < g.rows_out);
  }
}

template <typename T, bool ANY>
__global__ void __launch_bounds__(kMxThreads, kMxBlocks<ANY>)
mx_dequantize_kernel(const uint8_t* __restrict__ codes, const MxScales scales, const MxGrid g, T* __restrict__ y) {
  constexpr int E = Piece<T>::E;
  __shared__ __align__(16) uint8_t stage[ANY ? kMxThreads / 32 : 1][ANY ? kWarpStage : 1];
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const int G = min(g.lanes_x, 32);
  const int lane_x = threadIdx.x & (g.lanes_x - 1), lane = lane_x & (G - 1);
  const int col = (static_cast<int>(blockIdx.x) * g.lanes_x + lane_x) * E, first = col - lane * E;
  const int b = col / kMxBlock;
  const size_t pitch = static_cast<size_t>(scales.blocks) * 16;
  const size_t step = static_cast<size_t>(gridDim.y) * (kMxThreads >> g.log_x);
  uint8_t* my_stage = stage[ANY ? threadIdx.x >> 5 : 0];
  const Extent of_y = Extent::of(y, (g.rows - 1) * g.ld + g.K), of_codes = Extent::of(codes, g.rows * pitch);
  const size_t warp_row = (threadIdx.x & ~31u) >> g.log_x, my_row = (threadIdx.x >> g.log_x) - warp_row;
  for (size_t base = blockIdx.y * static_cast<size_t>(kMxThreads >> g.log_x) + warp_row; base < g.rows; base += step) {
    const size_t r = base + my_row;
    uint2 w = make_uint2(0u, 0u);
    uint32_t s = kScaleOne;
    const size_t at = r * pitch + col / 2;
    const size_t sat = scales.tiles ? mx_tile_word(r, b >> 2, scales.tiles_k) + (b & 3) : r * static_cast<size_t>(scales.blocks) + b;
    if (r < g.rows && b < scales.blocks && QC_AT(of_codes, codes + at, E / 2) && QC_IN(sat, scales.extent)) {
      if constexpr (E == 8) w.x = __ldg(reinterpret_cast<const uint32_t*>(codes + at));
      else w = __ldg(reinterpret_cast<const uint2*>(codes + at));
      s = __ldg(scales.bytes + sat);
    }
    float v[E];
    mx_decode_eight(w.x, scale_of(s), v);
    if constexpr (E == 16) mx_decode_eight(w.y, scale_of(s), v + 8);
    Piece<T> p;
    p.pack(v);
    group_store<ANY>(p, y + r * g.ld + first, r < g.rows ? g.K - first : 0, G, lane, g.unit, my_stage, of_y);
  }
}

}  // namespace qc
