// Entry points of the operators on microscaled 4-bit tensors, norms and caches (include/qconv.h): argument checks, plans
// and launches.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <mutex>
#include <new>

#include "../../include/qconv.h"
#include "kernel_mx_gemm.cuh"
#include "kernel_mx_gemm_pair.cuh"
#include "kernels_cache.cuh"
#include "kernels_mx.cuh"
#include "kernels_norm.cuh"
#include "library.cuh"
#include "per_device.cuh"
#include "status_words.cuh"

// The header's numbers and the kernels'.
constexpr int kOfHeader[] = {QTYPE_F32, QTYPE_BF16, QTYPE_F16, QNORM_I8, QNORM_I8_ROWS, QNORM_MX, QCACHE_I8, QCACHE_MX};
constexpr int kOfKernels[] = {qc::TYPE_F32, qc::TYPE_BF16, qc::TYPE_F16, qc::NORM_I8, qc::NORM_I8_ROWS, qc::NORM_MX, qc::CACHE_I8, qc::CACHE_MX};
constexpr bool same_numbers() {
  for (int i = 0; i < 8; ++i)
    if (kOfHeader[i] != kOfKernels[i]) return false;
  return true;
}
static_assert(same_numbers());

using qc::fail;
using qc::launch_chained;
using qc::make_fastdiv;

namespace {

constexpr long long kMaxRows = 1ll << 40;
constexpr long long kMaxUnits = 1ll << 30;        // pieces of a tensor that one launch counts in 31 bits

size_t type_size(int type) { return type == QTYPE_F32 ? 4 : 2; }
bool aligned(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

// Calls f with a value of the type that `type` stands for.
template <typename F>
auto with_type(int type, F&& f) {
  if (type == QTYPE_BF16) return f(__nv_bfloat16());
  if (type == QTYPE_F16) return f(__half());
  return f(float());
}
bool type_ok(int type) { return type == QTYPE_F32 || type == QTYPE_BF16 || type == QTYPE_F16; }

int check_mx(long long rows, int K, int layout) {
  if (rows <= 0 || K <= 0) return fail(QCONV_ERR_BAD_ARG, "rows and K must be positive");
  if (layout != QMX_ROWS && layout != QMX_TILES) return fail(QCONV_ERR_BAD_ARG, "unknown layout of scales %d", layout);
  if (rows > kMaxRows || K > (1 << 28)) return fail(QCONV_ERR_UNSUPPORTED_SHAPE, "tensor too large");
  const long long padded = layout == QMX_TILES ? (rows + 127) / 128 * 128 : rows;
  if (padded * ((K + 127ll) / 128) > kMaxUnits) return fail(QCONV_ERR_UNSUPPORTED_SHAPE, "tensor too large: more than 2^30 pieces of 128 values");
  return QCONV_OK;
}

size_t scale_bytes(long long rows, int K, int layout) {
  return layout == QMX_TILES ? static_cast<size_t>((rows + 127) / 128) * qc::mx_tiles_k(K) * qc::kMxTileBytes
                             : static_cast<size_t>(rows) * qc::mx_blocks(K);
}

qc::MxScales make_scales(uint8_t* bytes, long long rows, int K, int layout) {
  return {bytes, layout == QMX_TILES, qc::mx_blocks(K), qc::mx_tiles_k(K), scale_bytes(rows, K, layout)};
}

int check_code_alignment(const void* codes, const void* scales, int layout) {
  if (!aligned(codes, 16)) return fail(QCONV_ERR_ALIGNMENT, "codes must be 16-byte aligned");
  if (layout == QMX_TILES && !aligned(scales, 16)) return fail(QCONV_ERR_ALIGNMENT, "scales in tiles must be 16-byte aligned");
  return QCONV_OK;
}

int check_values(const void* p, int type, long long ld, int width, const char* what) {
  if (ld < width) return fail(QCONV_ERR_BAD_ARG, "row stride of %s is below the row's length", what);
  if (ld > kMaxRows) return fail(QCONV_ERR_UNSUPPORTED_SHAPE, "row stride of %s too large", what);
  if (!aligned(p, type_size(type))) return fail(QCONV_ERR_ALIGNMENT, "%s must be aligned to its type", what);
  return QCONV_OK;
}
// The unit, in bytes, that rows from p on, `ld` elements apart, may be reached in.
int reach(const void* p, int type, long long ld) {
  const uintptr_t bits = reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(ld * static_cast<long long>(type_size(type))) | 32u;
  return static_cast<int>(bits & (~bits + 1));               // the lowest bit
}

// The blocks of a conversion over `rows_out` rows: enough lanes along the row, and rows until the device is full.  any: lanes
// exchange values, as units below `own` bytes need it.
qc::MxGrid mx_grid(long long rows, long long rows_out, int K, long long ld, int type, const void* values, int own, dim3* grid, bool* any) {
  const int E = 32 / static_cast<int>(type_size(type));
  const int lanes = qc::mx_blocks(K) * (qc::kMxBlock / E);
  qc::MxGrid g = {};
  g.lanes_x = 128 / E;                                     // of a scale word
  while (g.lanes_x < qc::kMxThreads && g.lanes_x < lanes) g.lanes_x *= 2;
  while (g.lanes_x > 32 && ((lanes + g.lanes_x - 1) / g.lanes_x * g.lanes_x - lanes) * 8 > lanes) g.lanes_x /= 2;   // few lanes behind the row's end
  while ((1 << g.log_x) < g.lanes_x) ++g.log_x;
  g.rows = static_cast<size_t>(rows); g.rows_out = static_cast<size_t>(rows_out); g.K = K; g.ld = static_cast<size_t>(ld);
  g.unit = reach(values, type, ld);
  *any = g.unit < own;
  const long long per_block = qc::kMxThreads / g.lanes_x;
  grid->x = static_cast<unsigned int>((lanes + g.lanes_x - 1) / g.lanes_x);
  const long long most = std::max(1ll, 148ll * (*any ? qc::kMxBlocks<true> : qc::kMxBlocks<false>) / grid->x);   // (all at once, as many rows each)
  grid->y = static_cast<unsigned int>(std::min({(rows_out + per_block - 1) / per_block, most, 65535ll}));
  return g;
}

}  // namespace

namespace qc {
cudaError_t mx_checked_faults(int (&v)[2]) {
  v[0] = v[1] = 0;
#ifdef QCONV_CHECKED
  cudaError_t e = cudaMemcpyFromSymbol(v, g_checked_fault, sizeof(v));
  const int zero[2] = {0, 0};
  if (e == cudaSuccess) e = cudaMemcpyToSymbol(g_checked_fault, zero, sizeof(zero));
  return e;
#else
  return cudaSuccess;
#endif
}
}  // namespace qc

extern "C" {

// --------------------------------------------------------------------------- microscaled tensors
size_t qmx_code_bytes(long long rows, int K) {
  return rows <= 0 || K <= 0 ? 0 : static_cast<size_t>(rows) * qc::mx_blocks(K) * 16;
}

size_t qmx_scale_bytes(long long rows, int K, int layout) {
  if (rows <= 0 || K <= 0 || (layout != QMX_ROWS && layout != QMX_TILES)) return 0;
  return scale_bytes(rows, K, layout);
}

int qmx_quantize(const void* d_x, int type, long long rows, int K, long long ld, int rule, int layout, uint8_t* d_codes,
                 uint8_t* d_scales, void* cuda_stream) {
  if (!d_x || !d_codes || !d_scales) return fail(QCONV_ERR_BAD_ARG, "NULL tensor pointer");
  if (!type_ok(type)) return fail(QCONV_ERR_BAD_ARG, "unknown type %d", type);
  if (rule != QMX_COVER && rule != QMX_FLOOR) return fail(QCONV_ERR_BAD_ARG, "unknown rule %d", rule);
  int rc = check_mx(rows, K, layout);
  if (!rc) rc = check_values(d_x, type, ld, K, "x");
  if (!rc) rc = check_code_alignment(d_codes, d_scales, layout);
  if (rc) return rc;
  dim3 grid;
  bool any;
  const qc::MxGrid g = mx_grid(rows, layout == QMX_TILES ? (rows + 127) / 128 * 128 : rows, K, ld, type, d_x, qc::kLoadUnit, &grid, &any);
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    const auto kernel = any ? qc::mx_quantize_kernel<T, true> : qc::mx_quantize_kernel<T, false>;
    CUDA_TRY(launch_chained(kernel, grid, dim3(qc::kMxThreads), 0, static_cast<cudaStream_t>(cuda_stream), static_cast<const T*>(d_x), g, d_codes,
                            make_scales(d_scales, rows, K, layout), rule == QMX_COVER ? qc::kCoverRoundUp : 0u));
    return static_cast<int>(QCONV_OK);
  });
}

int qmx_dequantize(const uint8_t* d_codes, const uint8_t* d_scales, long long rows, int K, int layout, void* d_y, int type, long long ld,
                   void* cuda_stream) {
  if (!d_y || !d_codes || !d_scales) return fail(QCONV_ERR_BAD_ARG, "NULL tensor pointer");
  if (!type_ok(type)) return fail(QCONV_ERR_BAD_ARG, "unknown type %d", type);
  int rc = check_mx(rows, K, layout);
  if (!rc) rc = check_values(d_y, type, ld, K, "y");
  if (!rc) rc = check_code_alignment(d_codes, d_scales, layout);
  if (rc) return rc;
  dim3 grid;
  bool any;
  const qc::MxGrid g = mx_grid(rows, rows, K, ld, type, d_y, qc::kStoreUnit, &grid, &any);
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    const auto kernel = any ? qc::mx_dequantize_kernel<T, true> : qc::mx_dequantize_kernel<T, false>;
    CUDA_TRY(launch_chained(kernel, grid, dim3(qc::kMxThreads), 0, static_cast<cudaStream_t>(cuda_stream), d_codes,
                            make_scales(const_cast<uint8_t*>(d_scales), rows, K, layout), g, static_cast<T*>(d_y)));
    return static_cast<int>(QCONV_OK);
  });
}

// --------------------------------------------------------------------------- products
}  // extern "C"

static qc::StatusWords& status_words() {
  static qc::StatusWords* w = new qc::StatusWords;         // never destroyed, as the pool
  return *w;
}

struct qmx_linear {
  qmx_linear_desc d;
  const float* bias;
  DevicePool::Block block;               // of the status word where status_words() has none left
  int* d_status = nullptr;
  int device = 0, num_sms = 148;
  CUtensorMap map_w, map_ws;
  int bn = 0, split = 0, stages = 0;     // the last run's form
  int columns = 0;                       // of tensor memory, and bytes of shared memory of a CTA
  size_t smem = 0;
  bool pair = false, staged = false;
  unsigned int wait_limit = 1u << 22;
  cudaStream_t last_stream = nullptr;
  ~qmx_linear() {
    if (!d_status || block.ptr) return;
    // (whoever takes the word next must not see a status of this handle's)
    const qc::DeviceScope at(device);
    const bool idle = at.there && cudaDeviceSynchronize() == cudaSuccess;
    if (!idle) cudaGetLastError();                         // (no later call's)
    status_words().give(device, d_status, idle);
  }
};

namespace {

int encode_2d(CUtensorMap* map, CUtensorMapDataType type, const void* base, cuuint64_t inner, cuuint64_t rows, cuuint64_t pitch,
              cuuint32_t box_inner, cuuint32_t box_rows, CUtensorMapSwizzle swizzle) {
  const cuuint64_t dims[2] = {inner, rows}, strides[1] = {pitch};
  const cuuint32_t box[2] = {box_inner, box_rows}, steps[2] = {1, 1};
  return qc::encode_tiled(map, type, 2, base, dims, strides, box, steps, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
}
// Codes [rows][K] in boxes of `box_rows` rows x 256 values, and their scale tiles in boxes of two tiles along the
// contraction x those of `scale_rows` rows (what a box reaches beyond the arrays is read as zeros).
int encode_operand(CUtensorMap* codes, CUtensorMap* scales, const uint8_t* d_codes, const uint8_t* d_scales, int rows, int K, int box_rows, int scale_rows) {
  const cuuint64_t pitch = static_cast<cuuint64_t>(qc::mx_blocks(K)) * 16, tiles = qc::mx_tiles_k(K);
  int rc = encode_2d(codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, d_codes, pitch, rows, pitch, qc::kMxStageBytes, box_rows, CU_TENSOR_MAP_SWIZZLE_128B);
  if (!rc)
    rc = encode_2d(scales, CU_TENSOR_MAP_DATA_TYPE_UINT32, d_scales, tiles * 128, (rows + 127) / 128, tiles * qc::kMxTileBytes, 256,
                   (scale_rows + 127) / 128, CU_TENSOR_MAP_SWIZZLE_NONE);
  return rc;
}

// The tensor maps of one run's activations, their scales and (where it is stored in bulk) its output.
struct MxRunMaps { CUtensorMap x, xs, y; };

template <int BN, typename Y>
cudaError_t allow_gemm_smem() {
  return cudaFuncSetAttribute(qc::mx_gemm_kernel<BN, Y>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
}

template <int BN, typename Y>
int launch_gemm(qmx_linear* h, const MxRunMaps& maps, qc::MxGemmParams prm, Y* y, cudaStream_t st) {
  using Tile = qc::MxTile<BN>;
  static qc::PerDevice<cudaError_t> allowed;
  CUDA_TRY(allowed.once(h->device, allow_gemm_smem<BN, Y>));
  const int per_cta = (prm.k_stages + prm.split - 1) / prm.split;
  // Two CTAs an SM, so that one drains (or sets up, in the next launch) while the other multiplies; a deeper ring instead where
  // every CTA has an SM to itself and walks a long part of the contraction (us with half an SM's memory / all of it: 48 tokens x
  // 16384 x 8192 17.3 / 16.0, 128 x 8192 x 8192 16.5 / 13.6, 1 x 8192 x 28672 22.7 / 22.3; the other way round 64 x 4096 x 4096,
  // four stages a CTA, 5.3 / 6.0).  A shared tile's sums have shared memory of their own.
  const uint32_t sums = prm.split > 1 ? 16 + std::max(BN, 4 * prm.split) * 512 : 0;
  const bool alone = prm.tiles_n * prm.tiles_t * prm.split <= h->num_sms && per_cta >= 8;
  const uint32_t room = (alone ? 227u : 113u) * 1024 - 1024 - sizeof(qc::MxGemmShared) - sums;
  prm.stages = std::max(2, std::min({per_cta, static_cast<int>(room / Tile::kStage), Tile::kMaxStages}));
  const size_t smem = 1024 + static_cast<size_t>(prm.stages) * Tile::kStage + sizeof(qc::MxGemmShared) + sums;
  const unsigned int grid = static_cast<unsigned int>(prm.tiles_n) * prm.tiles_t * prm.split;
  const auto kernel = qc::mx_gemm_kernel<BN, Y>;
  h->bn = BN; h->split = prm.split; h->stages = prm.stages; h->pair = h->staged = false;
  h->columns = Tile::kCols; h->smem = prm.split > 1 ? qc::cluster_smem(smem, Tile::kCols) : smem;
  if (prm.split > 1)
    CUDA_TRY(qc::launch_clusters(kernel, grid, prm.split, qc::kMxGemmThreads, smem, Tile::kCols, qc::chained_launches(), st, h->map_w, maps.x,
                                 h->map_ws, maps.xs, prm, h->bias, y, h->d_status, h->wait_limit));
  else
    CUDA_TRY(launch_chained(kernel, dim3(grid), dim3(qc::kMxGemmThreads), smem, st, h->map_w, maps.x, h->map_ws, maps.xs, prm, h->bias, y,
                            h->d_status, h->wait_limit));
  return QCONV_OK;
}

template <typename Y, bool STAGED>
cudaError_t allow_pair_smem() {
  return cudaFuncSetAttribute(qc::mx_gemm_pair_kernel<Y, STAGED>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
}

template <typename Y, bool STAGED>
int launch_pair(qmx_linear* h, const MxRunMaps& maps, qc::MxGemmParams prm, Y* y, cudaStream_t st) {
  static qc::PerDevice<cudaError_t> allowed;
  CUDA_TRY(allowed.once(h->device, allow_pair_smem<Y, STAGED>));
  const unsigned int grid = 2u * std::min(prm.tiles_n * prm.tiles_t, h->num_sms / 2);
  const size_t smem = qc::kMxPairSmem<Y, STAGED>;
  const auto kernel = qc::mx_gemm_pair_kernel<Y, STAGED>;
  h->bn = qc::kMxPairTokens; h->split = 1; h->stages = qc::kMxPairStages; h->pair = true; h->staged = STAGED;
  h->columns = qc::kMxPairCols; h->smem = qc::cluster_smem(smem, qc::kMxPairCols);
  CUDA_TRY(qc::launch_clusters(kernel, grid, 2, qc::kMxPairThreads, smem, qc::kMxPairCols, qc::chained_launches(), st, h->map_w, maps.x,
                               h->map_ws, maps.xs, maps.y, prm, h->bias, y, h->d_status, h->wait_limit));
  return QCONV_OK;
}

}  // namespace

extern "C" {

int qmx_linear_create(qmx_linear** out, const qmx_linear_desc* desc, const uint8_t* d_w_codes, const uint8_t* d_w_scales, const float* d_bias) {
  if (!out) return fail(QCONV_ERR_BAD_ARG, "out is NULL");
  *out = nullptr;
  if (!desc || !d_w_codes || !d_w_scales) return fail(QCONV_ERR_BAD_ARG, "desc, d_w_codes or d_w_scales is NULL");
  if (!type_ok(desc->type)) return fail(QCONV_ERR_BAD_ARG, "unknown type %d", desc->type);
  int rc = check_mx(desc->N, desc->K, QMX_TILES);
  if (!rc) rc = check_code_alignment(d_w_codes, d_w_scales, QMX_TILES);
  if (rc) return rc;
  if (!aligned(d_bias, 4)) return fail(QCONV_ERR_ALIGNMENT, "the bias must be aligned to its type");
  qmx_linear* h = new (std::nothrow) qmx_linear();
  if (!h) return fail(QCONV_ERR_CUDA, "qmx_linear_create: out of host memory");
  h->d = *desc;
  h->bias = d_bias;
  rc = encode_operand(&h->map_w, &h->map_ws, d_w_codes, d_w_scales, desc->N, desc->K, 128, 128);
  cudaError_t e = cudaGetDevice(&h->device);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&h->num_sms, cudaDevAttrMultiProcessorCount, h->device);
  if (!rc && e == cudaSuccess) e = status_words().take(h->device, &h->d_status, [](int** base, size_t bytes) { return DevicePool::pool().plain(base, bytes); });
  if (!rc && e == cudaSuccess && !h->d_status) {
    e = DevicePool::pool().take(&h->block, sizeof(int));
    h->d_status = static_cast<int*>(h->block.ptr);
  }
  if (!rc && e == cudaSuccess) {
    const int zero = 0;
    e = cudaMemcpy(h->d_status, &zero, sizeof(int), cudaMemcpyHostToDevice);
  }
  if (!rc && e != cudaSuccess) rc = fail(QCONV_ERR_CUDA, "qmx_linear_create: %s", cudaGetErrorString(e));
  if (rc) { delete h; return rc; }
  *out = h;
  return QCONV_OK;
}

int qmx_linear_run(qmx_linear* h, const uint8_t* d_x_codes, const uint8_t* d_x_scales, int tokens, void* d_y, long long ld, void* cuda_stream) {
  if (!h || !d_x_codes || !d_x_scales || !d_y) return fail(QCONV_ERR_BAD_ARG, "NULL handle or tensor pointer");
  const qmx_linear_desc& d = h->d;
  int rc = check_mx(tokens, d.K, QMX_TILES);
  if (!rc) rc = check_code_alignment(d_x_codes, d_x_scales, QMX_TILES);
  if (!rc) rc = check_values(d_y, d.type, ld, d.N, "y");
  if (rc) return rc;
  int dev = 0;
  CUDA_TRY(cudaGetDevice(&dev));
  if (dev != h->device) return fail(QCONV_ERR_BAD_ARG, "the handle belongs to device %d, the current device is %d", h->device, dev);
  qc::MxGemmParams prm = {};
  prm.N = d.N; prm.T = tokens; prm.ld = static_cast<size_t>(ld); prm.relu = d.relu != 0;
  prm.k_tiles = qc::mx_tiles_k(d.K);
  prm.k_stages = (prm.k_tiles + 1) / 2;
  prm.tiles_n = (d.N + 127) / 128;
  const int bn_one = tokens <= 16 ? 16 : tokens <= 32 ? 32 : tokens <= 64 ? 64 : 128;
  const long long tiles_one = static_cast<long long>((d.N + 127) / 128) * ((tokens + bn_one - 1) / bn_one);
  const long long tiles_pair = static_cast<long long>((d.N + 255) / 256) * ((tokens + qc::kMxPairTokens - 1) / qc::kMxPairTokens);
  if (tiles_one > (1ll << 27)) return fail(QCONV_ERR_UNSUPPORTED_SHAPE, "product too large");
  // The form with the shortest estimate, in us without the launch.  Tiles on single SMs: 0.25 a stage and 0.35 for the output of
  // each round of tiles, two CTAs of an SM taking turns; sharing a tile 0.018 a column more.  On pairs: 0.33 a stage and round.  (us,
  // single / pair: 128 x 128 x 128 3.4 / 3.9, 700 x 700 x 700 4.2 / 4.8, 2048 x 2048 x 2048 7.8 / 9.1, 1024 x 4096 x 4096 11.5 / 13.8,
  // 384 x 8192 x 8192 18.2 / 15.0, 5555 x 422 x 152 6.1 / 5.3; shared by 1 / 2 / 4 / 8: 1 x 4096 x 4096 5.7 / 4.4 / 3.6 / 4.4,
  // 300 x 300 x 8192 10.7 / 8.7 / 6.7 / 6.3.)  More than two tiles an SM are pairs' (1000 x 5000 x 2000 17.1 / 11.5), but up to
  // 64 tokens a pair's columns are mostly empty.  Clusters of eight: sixteen of them with more than half an SM's memory a CTA do
  // not run at once (2025 x 64 x 2880 11.0, shared by four 5.8).
  const auto rounds = [&](long long tiles, int at_once) { return static_cast<double>((tiles + at_once - 1) / at_once); };
  double us_one = 0.0;
  for (int split = 1; split <= 8 && split <= prm.k_stages; split *= 2) {
    if (split > 1 && tiles_one * split > (split == 8 ? h->num_sms * 2 / 3 : h->num_sms)) break;
    const double us = (0.25 * ((prm.k_stages + split - 1) / split) + 0.35) * rounds(tiles_one * split, h->num_sms) + (split > 1 ? 0.018 * bn_one : 0.0);
    if (split == 1 || us < us_one) { us_one = us; prm.split = split; }
  }
  const double us_pair = 0.6 + 0.33 * prm.k_stages * rounds(tiles_pair, h->num_sms / 2);
  const bool pair = tokens > 64 && (tiles_one > 2 * h->num_sms || us_pair < us_one);
  const int bn = pair ? qc::kMxPairTokens : bn_one;
  if (pair) prm.tiles_n = (d.N + 255) / 256;
  prm.tiles_t = (tokens + bn - 1) / bn;
  MxRunMaps maps;
  rc = encode_operand(&maps.x, &maps.xs, d_x_codes, d_x_scales, tokens, d.K, pair ? bn / 2 : bn, pair ? 256 : bn);
  if (rc) return rc;
  // (bulk stores clip at 16 bytes along a row, not at its last value)
  const long long ysize = static_cast<long long>(type_size(d.type));
  const bool staged = pair && aligned(d_y, 16) && ld * ysize % 16 == 0 && d.N * ysize % 16 == 0;
  if (staged) {
    rc = encode_2d(&maps.y, d.type == QTYPE_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16, d_y, d.N, tokens,
                   static_cast<cuuint64_t>(ld * ysize), 128, 32, CU_TENSOR_MAP_SWIZZLE_NONE);
    if (rc) return rc;
  }
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  h->last_stream = st;
  return with_type(d.type, [&](auto t) {
    using Y = decltype(t);
    Y* y = static_cast<Y*>(d_y);
    if (pair) {
      return staged ? launch_pair<Y, true>(h, maps, prm, y, st) : launch_pair<Y, false>(h, maps, prm, y, st);
    }
    if (bn == 16) return launch_gemm<16, Y>(h, maps, prm, y, st);
    if (bn == 32) return launch_gemm<32, Y>(h, maps, prm, y, st);
    if (bn == 64) return launch_gemm<64, Y>(h, maps, prm, y, st);
    return launch_gemm<128, Y>(h, maps, prm, y, st);
  });
}

int qmx_linear_status(qmx_linear* h) {
  if (!h) return fail(QCONV_ERR_BAD_ARG, "NULL handle");
  const qc::DeviceScope at(h->device);                     // (the default stream is the current device's)
  if (!at.there) return fail(QCONV_ERR_CUDA, "qmx_linear_status: cannot make device %d current", h->device);
  CUDA_TRY(cudaStreamSynchronize(h->last_stream));
  int st = 0;
  CUDA_TRY(cudaMemcpy(&st, h->d_status, sizeof(int), cudaMemcpyDeviceToHost));
  if (st != 0) {
    CUDA_TRY(cudaMemset(h->d_status, 0, sizeof(int)));
    return fail(st, "a bounded device-side wait expired (status %d)", st);
  }
  return QCONV_OK;
}

int qmx_linear_set_wait_limit(qmx_linear* h, unsigned int polls) {
  if (!h) return fail(QCONV_ERR_BAD_ARG, "NULL handle");
  h->wait_limit = polls;
  return QCONV_OK;
}

int qmx_linear_describe(const qmx_linear* h, char* buf, size_t buf_len) {
  if (!h || !buf || buf_len == 0) return fail(QCONV_ERR_BAD_ARG, "NULL argument");
  snprintf(buf, buf_len, "mx N=%d K=%d tile=%dx%d split=%d pair=%d stages=%d staged=%d smem=%zu columns=%d", h->d.N, h->d.K, h->pair ? 256 : 128, h->bn, h->split,
           h->pair, h->stages, h->staged, h->smem, h->columns);
  return QCONV_OK;
}

int qmx_linear_destroy(qmx_linear* h) {
  if (!h) return fail(QCONV_ERR_BAD_ARG, "NULL handle");
  delete h;
  return QCONV_OK;
}

// --------------------------------------------------------------------------- norm
}  // extern "C"

namespace {

// Blocks that write the scale bytes of rows which only fill up the last tile.
template <int OUT, typename T>
unsigned int pad_blocks(const qc::NormArgs<T>& a) {
  if (OUT != qc::NORM_MX || !a.scales.tiles || a.rows % qc::kMxTileRows == 0) return 0;
  return static_cast<unsigned int>(std::min(16, (a.scales.tiles_k * qc::kMxTileRows + 1023) / 1024));
}

template <typename T, int OUT>
size_t norm_stages(const qc::NormArgs<T>& a, int warps) {
  return a.unit < qc::kLoadUnit || (OUT != qc::NORM_MX && !a.code_vec) ? static_cast<size_t>(warps) * qc::kWarpStage : 0;
}

// G lanes of a warp a row (four warps a block), or `warps` warps.
template <typename T, int OUT, int V>
int launch_norm(const qc::NormArgs<T>& a, int G, int warps, cudaStream_t st) {
  const unsigned int y = warps == 1 ? 4 : 1;
  const size_t per_block = static_cast<size_t>(y) * (32 / G);
  const unsigned int blocks = static_cast<unsigned int>((a.rows + per_block - 1) / per_block);
  auto kernel = qc::rmsnorm_kernel<T, OUT, V, false>;
  if constexpr (V <= 2) kernel = a.unit < qc::kLoadUnit ? qc::rmsnorm_kernel<T, OUT, V, true> : kernel;
  CUDA_TRY(launch_chained(kernel, dim3(blocks + pad_blocks<OUT>(a)), dim3(32 * warps, y), norm_stages<T, OUT>(a, warps * static_cast<int>(y)), st, a, G, blocks));
  return QCONV_OK;
}

// A row's values in registers: pieces of 32 bytes, one a lane for few rows (the more warps, the shorter the chain of a
// thread: one row of 4096 bf16 2.5 us, 3.0 with two, 5.6 with four), two for many (16384 x 8192 bf16 into 4 bits 140 us, 189
// with one, 154 with four; 134 since the sums over warps are shorter), four where a row is longer than two of every thread
// hold (rows that lanes exchange only up to two, which already take 80 registers).
template <typename T, int OUT>
int run_norm(const qc::NormArgs<T>& a, cudaStream_t st) {
  constexpr int E = qc::Piece<T>::E;
  const int lanes = (OUT == qc::NORM_MX ? qc::mx_blocks(a.C) * qc::kMxBlock : a.C + E - 1) / E;
  const auto warps = [&](int v) { return (lanes + 32 * v - 1) / (32 * v); };
  if (lanes <= 32) {
    int G = 128 / E;                                        // lanes of a scale word
    while (G < lanes) G *= 2;
    return launch_norm<T, OUT, 1>(a, G, 1, st);
  }
  // Two pieces a thread; one where rows are few, and where an odd number of warps takes one and the registers still leave
  // several rows an SM: up to three warps (16384 x 1536 bf16 to 4 bits 31.1 us against 33.3, 7021 x 3584 33.5 against 30.9);
  // where lanes exchange values, and two pieces take 80 registers, up to nine (5466 x 4604 bf16 40.4 against 48.5, 4911 x 5124
  // 54.9 against 51.4), or five in float32 (24504 x 1027 72.8 against 80.1, 14794 x 1701 67.3 against 67.2).
  const bool any = a.unit < qc::kLoadUnit, odd = warps(1) % 2 == 1 && warps(1) <= (!any ? 3 : sizeof(T) == 4 ? 5 : 9);
  if (lanes <= 1024 && (a.rows < 512 || odd)) return launch_norm<T, OUT, 1>(a, 32, warps(1), st);
  if (lanes <= 1024) return launch_norm<T, OUT, 2>(a, 32, warps(2), st);
  if (lanes <= 2048 && !any) return launch_norm<T, OUT, 4>(a, 32, warps(4), st);
  const auto kernel = any ? qc::rmsnorm_long_kernel<T, OUT, true> : qc::rmsnorm_long_kernel<T, OUT, false>;
  const unsigned int blocks = static_cast<unsigned int>(a.rows);
  CUDA_TRY(launch_chained(kernel, dim3(blocks + pad_blocks<OUT>(a)), dim3(32 * qc::kNormMaxWarps), norm_stages<T, OUT>(a, qc::kNormMaxWarps), st, a, blocks));
  return QCONV_OK;
}

}  // namespace

extern "C" {

int qrmsnorm(const qrmsnorm_args* args, void* cuda_stream) {
  if (!args) return fail(QCONV_ERR_BAD_ARG, "args is NULL");
  const qrmsnorm_args& g = *args;
  if (!g.d_x || !g.d_gain || !g.d_codes) return fail(QCONV_ERR_BAD_ARG, "NULL tensor pointer");
  if (!type_ok(g.type)) return fail(QCONV_ERR_BAD_ARG, "unknown type %d", g.type);
  if (g.out != QNORM_I8 && g.out != QNORM_I8_ROWS && g.out != QNORM_MX) return fail(QCONV_ERR_BAD_ARG, "unknown output %d", g.out);
  if (g.rows <= 0 || g.C <= 0) return fail(QCONV_ERR_BAD_ARG, "rows and C must be positive");
  if (g.rows > 0x7FFFFFFFll || g.C > (1 << 24)) return fail(QCONV_ERR_UNSUPPORTED_SHAPE, "tensor too large: rows below 2^31, C up to 2^24");
  if (!(g.eps >= 0.0) || std::isinf(g.eps)) return fail(QCONV_ERR_BAD_ARG, "eps must be finite and not negative");
  if (g.out == QNORM_I8 && (g.e < -126 || g.e > 126)) return fail(QCONV_ERR_BAD_ARG, "exponent %d outside [-126, 126]", g.e);
  if (g.out != QNORM_I8 && !g.d_scales) return fail(QCONV_ERR_BAD_ARG, "this output needs d_scales");
  int rc = check_values(g.d_x, g.type, g.ld_x, g.C, "x");
  if (!rc && g.d_residual) rc = check_values(g.d_residual, g.type, g.ld_residual, g.C, "the residual");
  if (!rc && g.d_sum) rc = check_values(g.d_sum, g.type, g.ld_sum, g.C, "the sum");
  if (!rc && !aligned(g.d_gain, type_size(g.type))) rc = fail(QCONV_ERR_ALIGNMENT, "the gain must be aligned to its type");
  if (!rc && g.out == QNORM_MX) {
    rc = check_mx(g.rows, g.C, g.layout);
    if (!rc) rc = check_code_alignment(g.d_codes, g.d_scales, g.layout);
  }
  if (rc) return rc;
  if (g.d_sum && ((g.d_sum == g.d_x && g.ld_sum != g.ld_x) || (g.d_sum == g.d_residual && g.ld_sum != g.ld_residual)))
    return fail(QCONV_ERR_BAD_ARG, "a sum in place of an input needs that input's row stride");
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  return with_type(g.type, [&](auto t) {
    using T = decltype(t);
    qc::NormArgs<T> a = {};
    a.x = static_cast<const T*>(g.d_x); a.residual = static_cast<const T*>(g.d_residual); a.gain = static_cast<const T*>(g.d_gain);
    a.sum = static_cast<T*>(g.d_sum);
    a.ld_x = g.ld_x; a.ld_res = g.d_residual ? g.ld_residual : 0; a.ld_sum = g.d_sum ? g.ld_sum : 0;
    a.rows = g.rows; a.C = g.C; a.eps = g.eps; a.inv_C = 1.0 / g.C;
    a.unit = reach(g.d_x, g.type, g.ld_x);
    a.unit_gain = reach(g.d_gain, g.type, 0);
    if (g.d_residual) a.unit = std::min(a.unit, reach(g.d_residual, g.type, g.ld_residual));
    if (g.d_sum) a.unit = std::min(a.unit, reach(g.d_sum, g.type, g.ld_sum));
    a.code_vec = aligned(g.d_codes, qc::Piece<T>::E) && g.C % qc::Piece<T>::E == 0;
    a.inv = std::ldexp(1.0f, -g.e);
    a.codes = g.d_codes;
    if (g.out == QNORM_MX) a.scales = make_scales(g.d_scales, g.rows, g.C, g.layout);
    else a.scales.bytes = g.d_scales;
    if (g.out == QNORM_I8) return run_norm<T, qc::NORM_I8>(a, st);
    if (g.out == QNORM_I8_ROWS) return run_norm<T, qc::NORM_I8_ROWS>(a, st);
    return run_norm<T, qc::NORM_MX>(a, st);
  });
}

// --------------------------------------------------------------------------- caches
}  // extern "C"

namespace {

// Checks and the kernels' arguments, the same for both directions.
int cache_args(const qcache_desc* c, const qcache_values* keys, const qcache_values* values, int type, const int64_t* d_slots, long long rows,
               qc::CacheArgs* a) {
  if (!c || !keys || !d_slots) return fail(QCONV_ERR_BAD_ARG, "cache, keys or d_slots is NULL");
  if (c->format != QCACHE_I8 && c->format != QCACHE_MX) return fail(QCONV_ERR_BAD_ARG, "unknown format %d", c->format);
  if (!type_ok(type)) return fail(QCONV_ERR_BAD_ARG, "unknown type %d", type);
  if (c->num_slots <= 0 || c->heads <= 0 || c->D <= 0 || rows < 0) return fail(QCONV_ERR_BAD_ARG, "num_slots, heads and D must be positive, rows not negative");
  if (c->D > 1024) return fail(QCONV_ERR_UNSUPPORTED_SHAPE, "D is at most 1024");
  if (c->heads > (1 << 20) || c->num_slots > (1ll << 40)) return fail(QCONV_ERR_UNSUPPORTED_SHAPE, "cache too large");
  a->sides = values ? 2 : 1;
  if (rows > kMaxUnits / c->heads / a->sides) return fail(QCONV_ERR_UNSUPPORTED_SHAPE, "more than 2^30 heads in one call");
  if (!aligned(d_slots, 8)) return fail(QCONV_ERR_ALIGNMENT, "slots must be aligned to their type");
  a->slots = reinterpret_cast<const long long*>(d_slots);
  a->num_slots = c->num_slots; a->heads = c->heads; a->D = c->D; a->blocks = qc::mx_blocks(c->D);
  a->items = static_cast<int>(rows * c->heads * a->sides);
  a->fd_heads = make_fastdiv(c->heads);
  a->code_pitch = c->format == QCACHE_I8 ? c->D : a->blocks * 16;
  a->scale_pitch = c->format == QCACHE_I8 ? 1 : a->blocks;
  const int per_lane = 32 / static_cast<int>(type_size(type));
  a->unit = 32;
  a->code_vec = c->D % per_lane == 0;
  const qcache_values* in[2] = {keys, values};
  uint8_t* codes[2] = {c->d_k_codes, c->d_v_codes};
  uint8_t* scales[2] = {c->d_k_scales, c->d_v_scales};
  for (int i = 0; i < a->sides; ++i) {
    const qcache_values& v = *in[i];
    if (!v.d_values || !codes[i] || !scales[i]) return fail(QCONV_ERR_BAD_ARG, "NULL tensor pointer");
    if (v.token_stride < 0 || v.head_stride < 0 || v.token_stride > kMaxRows || v.head_stride > kMaxRows)
      return fail(QCONV_ERR_BAD_ARG, "strides must not be negative, nor above 2^40");
    if (!aligned(v.d_values, type_size(type))) return fail(QCONV_ERR_ALIGNMENT, "values must be aligned to their type");
    if (c->format == QCACHE_MX && !aligned(codes[i], 16)) return fail(QCONV_ERR_ALIGNMENT, "codes must be 16-byte aligned");
    a->side[i] = {codes[i], scales[i], v.d_values, v.token_stride, v.head_stride};
    a->unit = std::min({a->unit, reach(v.d_values, type, v.token_stride), reach(v.d_values, type, v.head_stride)});
    a->code_vec &= aligned(codes[i], per_lane);
  }
  return QCONV_OK;
}

template <typename T, int FMT, int LANES, int V>
int launch_cache(const qc::CacheArgs& a, bool write, cudaStream_t st) {
  const bool any = write ? a.unit < qc::kLoadUnit || (FMT == qc::CACHE_I8 && !a.code_vec) : a.unit < qc::kStoreUnit;
  const auto kernel = write ? (any ? qc::cache_write_kernel<T, FMT, LANES, V, true> : qc::cache_write_kernel<T, FMT, LANES, V, false>)
                            : (any ? qc::cache_read_kernel<T, FMT, LANES, V, true> : qc::cache_read_kernel<T, FMT, LANES, V, false>);
  CUDA_TRY(launch_chained(kernel, dim3(qc::grid_for(a.items, qc::kCacheThreads / 32 * (32 / (any || !write ? LANES : a.lanes)), 148 * 8)), dim3(qc::kCacheThreads), 0, st, a));
  return QCONV_OK;
}
template <typename T, int FMT>
int run_cache(qc::CacheArgs a, bool write, cudaStream_t st) {
  const int lanes = (FMT == qc::CACHE_MX ? a.blocks * qc::kMxBlock : a.D) / qc::Piece<T>::E + (FMT == qc::CACHE_I8 && a.D % qc::Piece<T>::E != 0);
  a.lanes = lanes <= 2 ? 4 : std::min(lanes, 32);            // (above half of the forms' lanes, and whole blocks of 4-bit codes)
  if (lanes <= 4) return launch_cache<T, FMT, 4, 1>(a, write, st);
  if (lanes <= 8) return launch_cache<T, FMT, 8, 1>(a, write, st);
  if (lanes <= 16) return launch_cache<T, FMT, 16, 1>(a, write, st);
  if (lanes <= 32) return launch_cache<T, FMT, 32, 1>(a, write, st);
  return launch_cache<T, FMT, 32, 4>(a, write, st);
}
int run_cache(const qcache_desc* c, const qcache_values* keys, const qcache_values* values, int type, const int64_t* d_slots, long long rows,
              bool write, void* cuda_stream) {
  qc::CacheArgs a = {};
  const int rc = cache_args(c, keys, values, type, d_slots, rows, &a);
  if (rc || a.items == 0) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    return c->format == QCACHE_I8 ? run_cache<T, qc::CACHE_I8>(a, write, st) : run_cache<T, qc::CACHE_MX>(a, write, st);
  });
}

}  // namespace

extern "C" {

int qcache_write(const qcache_desc* cache, const qcache_values* keys, const qcache_values* values, int type, const int64_t* d_slots,
                 long long rows, void* cuda_stream) {
  return run_cache(cache, keys, values, type, d_slots, rows, true, cuda_stream);
}

int qcache_read(const qcache_desc* cache, const int64_t* d_slots, long long rows, const qcache_values* keys, const qcache_values* values,
                int type, void* cuda_stream) {
  return run_cache(cache, keys, values, type, d_slots, rows, false, cuda_stream);
}

}  // extern "C"
