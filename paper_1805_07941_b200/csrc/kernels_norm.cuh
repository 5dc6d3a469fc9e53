// Residual addition, root-mean-square norm and conversion to 8 or 4 bits, one pass:
//   h = x + residual rounded to the tensors' type (what the next residual addition reads is what is normalised here)
//   r = 1 / sqrt(mean(h^2) + eps), the sum and the root in 64 bits, r rounded to 32
//   y = (h r) gain in 32 bits, two rounded products
// and y to int8 at a given exponent, to int8 at the row's own exponent, or to microscaled 4 bits.  The sum of squares is
// kept in 64 bits so that r, and with it every code, does not depend on the order of the summation: codes
// are whole numbers, and a last-bit difference in r would move those that lie next to a border.
//
// Bound by HBM: x, residual and h once, the codes once.  A row's values stay in registers from the load to the
// conversion: V pieces of 32 bytes a thread, and as many lanes or warps as that makes for the row's length.  16384 x 8192 bf16
// with a residual into 4 bits: 134 us, the measured copy rate; rows whose pieces are not aligned pass through shared memory
// (12264 x 2052 bf16 into 4 bits 47 us, 12282 x 2049 65).
#pragma once
#include "mx_format.cuh"
#include "kernel_igemm.cuh"

namespace qc {

enum : int { NORM_I8 = 0, NORM_I8_ROWS = 1, NORM_MX = 2 };
constexpr int kNormMaxWarps = 32;

template <typename T>
struct NormArgs {
  const T* x;
  const T* residual;      // or null
  const T* gain;
  T* sum;                 // or null; may be x or residual
  size_t ld_x, ld_res, ld_sum, rows;
  int C, unit, unit_gain; // bytes that rows of x, residual and sum, and the gain, may be reached in
  int code_vec;           // a lane's int8 codes are aligned
  double eps, inv_C;
  float inv;              // NORM_I8: 2^-e
  uint8_t* codes;
  MxScales scales;        // NORM_I8_ROWS: bytes alone
};

// A tensor of a call, for the checked build: rows `ld` apart of C values (x, residual, sum), or what the outputs hold.
template <typename T> __device__ __forceinline__ Extent norm_extent(const NormArgs<T>& a, const T* p, size_t ld) {
  return Extent::of(p, (a.rows - 1) * ld + a.C);
}

// How the threads share out rows: a row is G lanes of a warp (a power of two, at least those of a scale word), or all of the
// block's warps (G = 32).
struct NormPlace {
  size_t row;
  int G, lane;            // lane within the group
  int warp, warps;        // warps of the row
  bool valid;
};

// Sum and maximum over a row; all of its threads get them.
__device__ __forceinline__ double row_sum(double v, double* shared, const NormPlace& at) {
  for (int d = at.G >> 1; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  if (at.warps > 1) {
    if (at.lane == 0) shared[at.warp] = v;
    __syncthreads();
    const int last = at.warps - 1, own = at.lane & (0x7FFFFFFF >> __clz(last) | last);
    v = own <= last ? shared[own] : 0.0;
    for (int d = 1; d <= last; d *= 2) v += __shfl_xor_sync(0xffffffffu, v, d);
  }
  return v;
}
__device__ __forceinline__ uint32_t row_max(uint32_t m, uint32_t* shared, const NormPlace& at) {
  for (int d = at.G >> 1; d > 0; d >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, d));
  if (at.warps > 1) {
    if (at.lane == 0) shared[at.warp] = m;
    __syncthreads();
    m = __reduce_max_sync(0xffffffffu, at.lane < at.warps ? shared[at.lane] : 0u);
  }
  return m;
}

// What a lane has loaded of x and the residual, before it is added up (ANY: as the lanes share it out).
template <typename T> struct NormRaw {
  Piece<T> x, r;
  uint32_t x_ends, r_ends;                                  // (rows moved by bytes)
};

// The group's pieces from column `first` on: loaded (all of a thread's loads come before the first use) ...
template <bool ANY, typename T>
__device__ __forceinline__ void norm_fetch(const NormArgs<T>& a, const NormPlace& at, int first, NormRaw<T>& raw) {
  const int n = at.valid ? a.C - first : 0;
  const T* px = a.x + at.row * a.ld_x + first;
  const T* pr = a.residual + at.row * a.ld_res + first;
  const Extent of_x = norm_extent(a, a.x, a.ld_x), of_r = norm_extent(a, a.residual, a.ld_res);
  if constexpr (ANY) {
    if (by_bytes<T>(a.unit)) {
      load_piece(raw.x, raw.x_ends, px, n, at.G, at.lane, of_x);
      if (a.residual) load_piece(raw.r, raw.r_ends, pr, n, at.G, at.lane, of_r);
    } else {
      with_unit(a.unit, [&](auto u) {
        load_dealt<decltype(u)::value>(raw.x, px, n, at.G, at.lane, of_x);
        if (a.residual) load_dealt<decltype(u)::value>(raw.r, pr, n, at.G, at.lane, of_r);
      });
    }
  } else {
    group_load<false>(raw.x, px, n, at.G, at.lane, a.unit, nullptr, of_x);
    if (a.residual) group_load<false>(raw.r, pr, n, at.G, at.lane, a.unit, nullptr, of_r);
  }
}
template <typename T> __device__ __forceinline__ void add_residual(Piece<T>& h, const Piece<T>& residual) {
  float v[Piece<T>::E], u[Piece<T>::E];
  h.unpack(v);
  residual.unpack(u);
#pragma unroll
  for (int i = 0; i < Piece<T>::E; ++i) v[i] += u[i];
  h.pack(v);                                                // (the rounding to T)
}
// ... and h of them: added, rounded, kept.
template <bool ANY, typename T>
__device__ __forceinline__ void norm_add(const NormArgs<T>& a, const NormPlace& at, int first, NormRaw<T>& raw, Piece<T>& h, uint8_t* stage) {
  const int n = at.valid ? a.C - first : 0;
  T* ps = a.sum + at.row * a.ld_sum + first;
  const Extent of_s = norm_extent(a, a.sum, a.ld_sum);
  if (ANY && by_bytes<T>(a.unit)) {                         // (the three may begin at different bytes of a word)
    gather_piece(raw.x, raw.x_ends, a.x + at.row * a.ld_x + first, n, at.G, at.lane, stage);
    h = raw.x;
    if (a.residual) {
      gather_piece(raw.r, raw.r_ends, a.residual + at.row * a.ld_res + first, n, at.G, at.lane, stage);
      add_residual(h, raw.r);
    }
    if (a.sum) store_piece(h, ps, n, at.G, at.lane, stage, of_s);
    return;
  }
  h = raw.x;
  if (a.residual) add_residual(h, raw.r);
  if constexpr (ANY) {
    with_unit(a.unit, [&](auto u) {
      if (a.sum) store_dealt<decltype(u)::value>(h, ps, n, at.G, at.lane, of_s);
      gather_dealt<decltype(u)::value>(h, at.G, at.lane, stage);
    });
  } else {
    if (a.sum) group_store<false>(h, ps, n, at.G, at.lane, a.unit, nullptr, of_s);
  }
}

template <typename T>
__device__ __forceinline__ double add_squares(const Piece<T>& h, double sum) {
  float v[Piece<T>::E];
  h.unpack(v);
#pragma unroll
  for (int i = 0; i < Piece<T>::E; ++i) sum = fma(static_cast<double>(v[i]), static_cast<double>(v[i]), sum);
  return sum;
}

// y of those pieces (zeros behind the row's end).
template <typename T>
__device__ __forceinline__ void norm_scale(const NormArgs<T>& a, const NormPlace& at, int first, float r, const Piece<T>& h, float (&y)[Piece<T>::E]) {
  constexpr int E = Piece<T>::E;
  Piece<T> g;
  float u[E];
  const Extent of_g = Extent::of(a.gain, a.C);
  if (a.unit_gain >= kLoadUnit) {
    group_load<false>(g, a.gain + first, a.C - first, at.G, at.lane, a.unit_gain, nullptr, of_g);
    g.unpack(u);
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int c = first + at.lane * E + i;
      u[i] = c < a.C && QC_AT(of_g, a.gain + c, sizeof(T)) ? to_float(a.gain[c]) : 0.0f;
    }
  }
  h.unpack(y);
#pragma unroll
  for (int i = 0; i < E; ++i) y[i] = (y[i] * r) * u[i];
}

template <typename T>
__device__ __forceinline__ void norm_store_i8(const NormArgs<T>& a, const NormPlace& at, int first, const float (&y)[Piece<T>::E], float inv, uint8_t* stage) {
  constexpr int E = Piece<T>::E;
  const int n = at.valid ? a.C - first : 0;
  uint32_t c[E / 4];
#pragma unroll
  for (int i = 0; i < E / 4; ++i) c[i] = i8_encode_four(y + 4 * i, inv);
  uint8_t* p = a.codes + at.row * a.C + first;
  const Extent of_codes = Extent::of(a.codes, a.rows * a.C);
  if (a.code_vec) {                                         // (C is then a multiple of E, too)
    if (at.lane * E >= n || !QC_AT(of_codes, p + at.lane * E, E)) return;
    if constexpr (E == 8) *reinterpret_cast<uint2*>(p + at.lane * E) = make_uint2(c[0], c[1]);
    else *reinterpret_cast<uint4*>(p + at.lane * E) = make_uint4(c[0], c[1], c[2], c[3]);
  } else {
    uint8_t* mine = stage + ((threadIdx.x & 31) - at.lane) * E;
#pragma unroll
    for (int i = 0; i < E / 4; ++i) reinterpret_cast<uint32_t*>(mine)[at.lane * (E / 4) + i] = c[i];
    __syncwarp();
    store_bytes<E>(p, mine, min(n, at.G * E), at.G, at.lane, of_codes);
    __syncwarp();
  }
}

template <typename T>
__device__ __forceinline__ void norm_store_mx(const NormArgs<T>& a, const NormPlace& at, int first, float (&y)[Piece<T>::E]) {
  constexpr int E = Piece<T>::E, kBlockLanes = kMxBlock / E;
  const int col = first + at.lane * E;
  const uint32_t s = mx_scale_byte(finite_top<kBlockLanes>(y, top_bits(y)), kCoverRoundUp);
  const int padded = a.scales.blocks * kMxBlock;
  const bool here = at.valid && col < padded;
  store_scale<kBlockLanes>(a.scales, at.row, col, s, here);
  if (here)
    mx_store_codes(a.codes + at.row * static_cast<size_t>(padded / 2) + col / 2, y, inverse_scale(s), Extent::of(a.codes, a.rows * (padded / 2)));
}

// Scale words of the rows that fill up the last tile of 128, by `blocks` blocks of which this is number `block`.
template <typename T>
__device__ __forceinline__ void norm_pad_rows(const NormArgs<T>& a, int block, int blocks) {
  const size_t tile0 = (a.rows - 1) & ~static_cast<size_t>(kMxTileRows - 1);
  const int real = static_cast<int>(a.rows - tile0), threads = blockDim.x * blockDim.y;
  // word i of the last row of tiles is word i % 128 of tile i / 128, and that is row i % 128 / 4 + 32 (i % 4)
  const int words = a.scales.tiles_k * kMxTileRows;
  for (int i = block * threads + threadIdx.y * blockDim.x + threadIdx.x; i < words; i += blocks * threads) {
    const int r = (i & 127) >> 2 | (i & 3) << 5;
    if (r >= real) store_scale_word(a.scales, tile0 + r, i >> 7, 0x01010101u * kScaleOne);
  }
}

// r.  (1 / C from the host and the reciprocal root in one function, off by 2^-52 or so like the sum itself, take a tenth of the
// instructions of a division, a root and another division.)
template <typename T> __device__ __forceinline__ float norm_factor(const NormArgs<T>& a, double sum) {
  return static_cast<float>(rsqrt(fma(sum, a.inv_C, a.eps)));
}

// Blocks behind those of the rows (row_blocks of them) write the padding scale words.
template <typename T, int OUT, int V, bool ANY>
__global__ void __launch_bounds__(V == 1 ? 1024 : 512)
rmsnorm_kernel(const NormArgs<T> a, int G, unsigned int row_blocks) {
  constexpr int E = Piece<T>::E;
  __shared__ double sums[kNormMaxWarps];
  __shared__ uint32_t tops[kNormMaxWarps];
  extern __shared__ __align__(16) uint8_t stages[];         // kWarpStage a warp; none where everything is aligned
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  if constexpr (OUT == NORM_MX) {
    if (blockIdx.x >= row_blocks) { norm_pad_rows(a, blockIdx.x - row_blocks, gridDim.x - row_blocks); return; }
  }
  // the rows of a warp (blockDim.y warps a block), or one row a block
  NormPlace at;
  at.G = G; at.lane = threadIdx.x & (G - 1);
  at.warp = threadIdx.x >> 5; at.warps = blockDim.x >> 5;
  at.row = (static_cast<size_t>(blockIdx.x) * blockDim.y + threadIdx.y) * (32 / G) + (at.warps > 1 ? 0 : threadIdx.x / G);
  at.valid = at.row < a.rows;
  uint8_t* stage = stages + (at.warp + threadIdx.y) * kWarpStage;
  Piece<T> h[V];
  {
    NormRaw<T> raw[V];
#pragma unroll
    for (int v = 0; v < V; ++v) norm_fetch<ANY>(a, at, (v * at.warps + at.warp) * 32 * E, raw[v]);
#pragma unroll
    for (int v = 0; v < V; ++v) norm_add<ANY>(a, at, (v * at.warps + at.warp) * 32 * E, raw[v], h[v], stage);
  }
  double sum = 0.0;
#pragma unroll
  for (int v = 0; v < V; ++v) sum = add_squares(h[v], sum);
  const float r = norm_factor(a, row_sum(sum, sums, at));
  if constexpr (OUT == NORM_I8_ROWS) {
    float y[V][E];
    uint32_t m = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      norm_scale(a, at, (v * at.warps + at.warp) * 32 * E, r, h[v], y[v]);
      m = max(m, finite_top<1>(y[v], top_bits(y[v])));
    }
    const uint32_t s = i8_scale_byte(row_max(m, tops, at));
    if (at.lane == 0 && at.warp == 0 && at.valid && QC_IN(at.row, a.rows)) a.scales.bytes[at.row] = static_cast<uint8_t>(s);
#pragma unroll
    for (int v = 0; v < V; ++v) norm_store_i8(a, at, (v * at.warps + at.warp) * 32 * E, y[v], inverse_scale(s), stage);
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int first = (v * at.warps + at.warp) * 32 * E;
      float y[E];
      norm_scale(a, at, first, r, h[v], y);
      if constexpr (OUT == NORM_MX) norm_store_mx(a, at, first, y);
      else norm_store_i8(a, at, first, y, a.inv, stage);
    }
  }
}

// Rows longer than the registers of a block hold: one block a row, h read again (from where it was kept, by the thread that
// kept it, else made again) for each further step.
template <typename T, int OUT, bool ANY>
__global__ void __launch_bounds__(32 * kNormMaxWarps)
rmsnorm_long_kernel(const NormArgs<T> a, unsigned int row_blocks) {
  constexpr int E = Piece<T>::E, kStep = kNormMaxWarps * 32 * E;
  __shared__ double sums[kNormMaxWarps];
  __shared__ uint32_t tops[kNormMaxWarps];
  extern __shared__ __align__(16) uint8_t stages[];
  ptx::grid_dependency_wait();
  ptx::grid_launch_dependents();
  if constexpr (OUT == NORM_MX) {
    if (blockIdx.x >= row_blocks) { norm_pad_rows(a, blockIdx.x - row_blocks, gridDim.x - row_blocks); return; }
  }
  const NormPlace at = {blockIdx.x, 32, static_cast<int>(threadIdx.x & 31), static_cast<int>(threadIdx.x >> 5), kNormMaxWarps, true};
  uint8_t* stage = stages + at.warp * kWarpStage;
  NormArgs<T> again = a;
  if (a.sum) { again.x = a.sum; again.ld_x = a.ld_sum; again.residual = nullptr; }
  again.sum = nullptr;
  Piece<T> h;
  NormRaw<T> raw;
  float y[E];
  double sum = 0.0;
  for (int first = at.warp * 32 * E; first < a.C; first += kStep) {
    norm_fetch<ANY>(a, at, first, raw);
    norm_add<ANY>(a, at, first, raw, h, stage);
    sum = add_squares(h, sum);
  }
  const float r = norm_factor(a, row_sum(sum, sums, at));
  float inv = a.inv;
  if constexpr (OUT == NORM_I8_ROWS) {
    uint32_t m = 0;
    for (int first = at.warp * 32 * E; first < a.C; first += kStep) {
      norm_fetch<ANY>(again, at, first, raw);
      norm_add<ANY>(again, at, first, raw, h, stage);
      norm_scale(a, at, first, r, h, y);
      m = max(m, finite_top<1>(y, top_bits(y)));
    }
    const uint32_t s = i8_scale_byte(row_max(m, tops, at));
    inv = inverse_scale(s);
    if (threadIdx.x == 0 && QC_IN(at.row, a.rows)) a.scales.bytes[at.row] = static_cast<uint8_t>(s);
  }
  for (int first = at.warp * 32 * E; first < a.C; first += kStep) {
    norm_fetch<ANY>(again, at, first, raw);
    norm_add<ANY>(again, at, first, raw, h, stage);
    norm_scale(a, at, first, r, h, y);
    if constexpr (OUT == NORM_MX) norm_store_mx(a, at, first, y);
    else norm_store_i8(a, at, first, y, inv, stage);
  }
}

}  // namespace qc
