// Residual addition, root-mean-square norm and conversion to 8 or 4 bits, one pass:
//   h = x + residual rounded to the tensors' type (what the next residual addition reads is what is normalised here)
//   r = 1 / sqrt(mean(h^2) + eps), the sum and the root in 64 bits, r rounded to 32
//   y = (h r) gain in 32 bits, two rounded products
// and y to int8 at a given exponent, to int8 at the row's own exponent, or to microscaled 4 bits.  The sum of squares is
// kept in 64 bits so that r, and with it every code, does not depend on the order of the summation: codes
// are whole numbers, and a last-bit difference in r would move those that lie next to a border.
//
// Bound by HBM: x, residual and h once, the codes once.  A row's values stay in registers from the load to the
// conversion: W warps a row with V vectors of eight values a thread.
#pragma once
#include "mx_format.cuh"
#include "kernel_igemm.cuh"

namespace qc {

enum : int { NORM_I8 = 0, NORM_I8_ROWS = 1, NORM_MX = 2 };

template <typename T>
struct NormArgs {
  const T* x;
  const T* residual;      // or null
  const T* gain;
  T* sum;                 // or null; may be x or residual
  size_t ld_x, ld_res, ld_sum, rows;
  int C, vec_ok, code_vec; // whole vectors of eight values are aligned; eight int8 codes are
  double eps;
  float inv;              // NORM_I8: 2^-e
  uint8_t* codes;
  MxScales scales;        // NORM_I8_ROWS: bytes alone
};

template <int W> constexpr int kNormThreads = W >= 4 ? 32 * W : 128;   // of a block

// Sum over a row's W warps; every thread gets it.
template <int W>
__device__ __forceinline__ double row_sum(double v, double* shared) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  if constexpr (W > 1) {
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
    __syncthreads();
    v = shared[threadIdx.x & (W - 1)];
#pragma unroll
    for (int d = W / 2; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  }
  return v;
}
template <int W>
__device__ __forceinline__ uint32_t row_max(uint32_t m, uint32_t* shared) {
  m = __reduce_max_sync(0xffffffffu, m);
  if constexpr (W > 1) {
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = m;
    __syncthreads();
    m = __reduce_max_sync(0xffffffffu, shared[threadIdx.x & (W - 1)]);
  }
  return m;
}

// h of the eight values from `col` on, n of them in the row: loaded, added, rounded, kept.
template <typename T>
__device__ __forceinline__ void norm_load(const NormArgs<T>& a, size_t row, int col, float (&h)[8]) {
  const int n = a.C - col;
  const T* px = a.x + row * a.ld_x + col;
  const T* pr = a.residual + row * a.ld_res + col;
  if (n >= 8 && a.vec_ok && QC_IN(row, a.rows)) {
    Eight<T> e, f;
    e.load_written(px);
    if (a.residual) f.load_written(pr);
    e.unpack(h);
    if (a.residual) {
      float g[8];
      f.unpack(g);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] += g[i];
      e.pack(h);                                            // (the rounding to T)
      e.unpack(h);
    }
    if (a.sum) e.store(a.sum + row * a.ld_sum + col);
  } else if (n > 0 && QC_IN(row, a.rows)) {
    load_some(px, n, h);
    if (a.residual) {
      float g[8];
      load_some(pr, n, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] = to_float(from_float<T>(h[i] + g[i]));
    }
    if (a.sum) store_some(a.sum + row * a.ld_sum + col, n, h);
  } else {
    load_some(px, 0, h);
  }
}

// y of those values (zeros behind the row's end).
template <typename T>
__device__ __forceinline__ void norm_scale(const NormArgs<T>& a, int col, float r, float (&h)[8]) {
  const int n = a.C - col;
  float g[8];
  if (n >= 8 && a.vec_ok) {
    Eight<T> e;
    e.load(a.gain + col);
    e.unpack(g);
  } else {
    load_some(a.gain + min(col, a.C), n, g);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) h[i] = (h[i] * r) * g[i];
}

template <typename T>
__device__ __forceinline__ void norm_store_i8(const NormArgs<T>& a, size_t row, int col, const float (&y)[8], float inv) {
  const int n = min(8, a.C - col);
  if (n <= 0 || !QC_IN(row, a.rows)) return;
  const uint2 c = i8_encode_eight(y, inv);
  uint8_t* p = a.codes + row * a.C + col;
  if (n == 8 && a.code_vec) *reinterpret_cast<uint2*>(p) = c;
  else
    for (int i = 0; i < n; ++i) p[i] = static_cast<uint8_t>((i < 4 ? c.x : c.y) >> (8 * (i & 3)));
}

// Whole warps: four lanes a block, sixteen a scale word.
template <typename T>
__device__ __forceinline__ void norm_store_mx(const NormArgs<T>& a, size_t row, int col, float (&y)[8]) {
  const uint32_t s = mx_scale_byte(finite_top<4>(y), 0x3FFFFFu);
  const uint32_t word = gather_scale_word(s);
  const int padded = a.scales.blocks * kMxBlock;
  if (!QC_IN(row, a.rows)) return;
  if (col < padded) *reinterpret_cast<uint32_t*>(a.codes + row * static_cast<size_t>(padded / 2) + col / 2) = mx_encode_eight(y, inverse_scale(s));
  if ((col & 127) == 0 && col < padded) store_scale_word(a.scales, row, col >> 7, word);
}

// Scale words of the rows that fill up the last tile of 128: shared out among the tile's real rows.
template <typename T>
__device__ __forceinline__ void norm_pad_rows(const NormArgs<T>& a, size_t row, int tid, int threads) {
  const size_t tile0 = (a.rows - 1) & ~static_cast<size_t>(kMxTileRows - 1);
  if (!a.scales.tiles || row < tile0) return;
  for (size_t p = a.rows + (row - tile0); p < tile0 + kMxTileRows; p += a.rows - tile0)
    for (int t = tid; t < a.scales.tiles_k; t += threads) store_scale_word(a.scales, p, t, 0x01010101u * kScaleOne);
}

__device__ __forceinline__ float norm_factor(double sum, int C, double eps) {
  return static_cast<float>(1.0 / sqrt(sum / C + eps));
}

template <typename T, int OUT, int W, int V>
__global__ void __launch_bounds__(kNormThreads<W>)
rmsnorm_kernel(const NormArgs<T> a) {
  __shared__ double sums[W];
  __shared__ uint32_t tops[W];
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  constexpr int kRows = kNormThreads<W> / (32 * W);       // rows of a block
  const int tid = W == 1 ? threadIdx.x & 31 : threadIdx.x;  // thread of the row
  const size_t row = static_cast<size_t>(blockIdx.x) * kRows + (W == 1 ? threadIdx.x >> 5 : 0);
  if (row >= a.rows) return;                                // (a whole warp, and only where a row is one warp)
  float h[V][8];
  double sum = 0.0;
#pragma unroll
  for (int v = 0; v < V; ++v) norm_load(a, row, (v * W * 32 + tid) * 8, h[v]);
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = fma(static_cast<double>(h[v][i]), static_cast<double>(h[v][i]), sum);
  const float r = norm_factor(row_sum<W>(sum, sums), a.C, a.eps);
#pragma unroll
  for (int v = 0; v < V; ++v) norm_scale(a, (v * W * 32 + tid) * 8, r, h[v]);
  if constexpr (OUT == NORM_MX) {
#pragma unroll
    for (int v = 0; v < V; ++v) norm_store_mx(a, row, (v * W * 32 + tid) * 8, h[v]);
    norm_pad_rows(a, row, tid, 32 * W);
  } else {
    float inv = a.inv;
    if constexpr (OUT == NORM_I8_ROWS) {
      uint32_t m = 0;
#pragma unroll
      for (int v = 0; v < V; ++v) m = max(m, finite_top<1>(h[v]));
      const uint32_t s = i8_scale_byte(row_max<W>(m, tops));
      inv = inverse_scale(s);
      if (tid == 0) a.scales.bytes[row] = static_cast<uint8_t>(s);
    }
#pragma unroll
    for (int v = 0; v < V; ++v) norm_store_i8(a, row, (v * W * 32 + tid) * 8, h[v], inv);
  }
}

// Rows longer than the registers of a block hold: one block a row, h read again (from where it was kept, else made again)
// for each further step.
constexpr int kNormLongWarps = 32;
template <typename T, int OUT>
__global__ void __launch_bounds__(32 * kNormLongWarps)
rmsnorm_long_kernel(const NormArgs<T> a) {
  __shared__ double sums[kNormLongWarps];
  __shared__ uint32_t tops[kNormLongWarps];
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  const size_t row = blockIdx.x;
  constexpr int kStep = kNormLongWarps * 32 * 8;
  const int first = threadIdx.x * 8;
  NormArgs<T> again = a;
  if (a.sum) { again.x = a.sum; again.ld_x = a.ld_sum; again.residual = nullptr; }
  again.sum = nullptr;
  float h[8];
  double sum = 0.0;
  for (int col = first; col - first < a.C; col += kStep) {
    norm_load(a, row, col, h);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = fma(static_cast<double>(h[i]), static_cast<double>(h[i]), sum);
  }
  const float r = norm_factor(row_sum<kNormLongWarps>(sum, sums), a.C, a.eps);
  float inv = a.inv;
  if constexpr (OUT == NORM_I8_ROWS) {
    uint32_t m = 0;
    for (int col = first; col - first < a.C; col += kStep) {
      norm_load(again, row, col, h);
      norm_scale(a, col, r, h);
      m = max(m, finite_top<1>(h));
    }
    const uint32_t s = i8_scale_byte(row_max<kNormLongWarps>(m, tops));
    inv = inverse_scale(s);
    if (threadIdx.x == 0) a.scales.bytes[row] = static_cast<uint8_t>(s);
  }
  for (int col = first; col - first < a.C; col += kStep) {
    norm_load(again, row, col, h);
    norm_scale(a, col, r, h);
    if constexpr (OUT == NORM_MX) norm_store_mx(a, row, col, h);
    else norm_store_i8(a, row, col, h, inv);
  }
  if constexpr (OUT == NORM_MX) norm_pad_rows(a, row, threadIdx.x, 32 * kNormLongWarps);
}

}  // namespace qc
