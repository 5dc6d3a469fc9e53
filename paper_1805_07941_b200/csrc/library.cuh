// What the translation units of the library share: error texts, tensor-map encoding, the pool of device memory, divisions
// prepared on the host, and launches that may start while the kernel before them drains.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>
#include <cstring>
#include <mutex>
#include <utility>
#include <vector>

#include "../../include/qconv.h"
#include "kernel_igemm.cuh"
#include "tensor_memory.cuh"

#define QC_HIDDEN __attribute__((visibility("hidden")))

namespace qc {

// Keeps the text for qconv_last_error_string (of the calling thread) and returns `code`.
QC_HIDDEN int fail(int code, const char* fmt, ...);

// Tensor map of `base`, not interleaved, zeros outside; QCONV_OK or an error with its text.  From any host thread.
QC_HIDDEN int encode_tiled(CUtensorMap* map, CUtensorMapDataType type, int rank, const void* base, const cuuint64_t* dims,
                           const cuuint64_t* strides_bytes, const cuuint32_t* box, const cuuint32_t* elem_strides, CUtensorMapSwizzle swizzle,
                           CUtensorMapL2promotion promotion);

// Whether the calling thread's plan hints leave programmatic dependent launch on.
QC_HIDDEN bool chained_launches();

// Failed index tests of the kernels in mx_api.cu (checked build), as qconv_checked_faults reports them; clears them.
QC_HIDDEN cudaError_t mx_checked_faults(int (&v)[2]);

// Multiplier and shift for the kernel's divisions by d (1 <= d < 2^31) of n < 2^31.  With 2^shr < d <= 2^(shr+1) and
// mul = ceil(2^(32+shr) / d), e = mul d - 2^(32+shr) lies in [0, d), so n e < 2^31 2^(shr+1) = 2^(32+shr): the quotient
// n mul / 2^(32+shr) exceeds n / d by less than 1 / d and has the same whole part.
inline FastDiv make_fastdiv(int d_in) {
  FastDiv f = {0u, 0u, static_cast<uint32_t>(std::max(1, d_in))};
  if (f.d > 1u) {
    uint32_t lg = 0;
    while ((1ull << lg) < f.d) ++lg;                       // ceil(log2 d) >= 1
    f.shr = lg - 1;
    f.mul = static_cast<uint32_t>(((1ull << (32 + f.shr)) + f.d - 1) / f.d);
  }
  return f;
}

// Launch with the programmatic-dependent-launch attribute (the kernel must wait for the kernels before it, griddepcontrol.wait, first).
template <typename... KArgs, typename... Args>
cudaError_t launch_chained(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = chained_launches() ? 1 : 0;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

// Launch in clusters of CTAs that allocate `columns` columns of tensor memory each; `chained` as above.
template <typename... KArgs, typename... Args>
cudaError_t launch_clusters(void (*kernel)(KArgs...), unsigned int grid, unsigned int cluster, unsigned int threads, size_t smem, int columns,
                            bool chained, cudaStream_t st, const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = cluster_smem(smem, columns);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = chained ? 1 : 0;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// Another device for a while: current from here to the end of the scope where `there`.
class DeviceScope {
 public:
  explicit DeviceScope(int device) {
    there = cudaGetDevice(&before_) == cudaSuccess && (before_ == device || (other_ = cudaSetDevice(device) == cudaSuccess));
  }
  ~DeviceScope() { if (other_) cudaSetDevice(before_); }
  DeviceScope(const DeviceScope&) = delete;
  DeviceScope& operator=(const DeviceScope&) = delete;
  bool there = false;

 private:
  int before_ = 0;
  bool other_ = false;
};

inline int grid_for(size_t work_items, int threads, int max_blocks) {
  size_t b = (work_items + threads - 1) / threads;
  return static_cast<int>(std::max<size_t>(1, std::min<size_t>(b, max_blocks)));
}

}  // namespace qc

#define CUDA_TRY(expr)                                                                        \
  do {                                                                                        \
    cudaError_t e_ = (expr);                                                                  \
    if (e_ != cudaSuccess)                                                                    \
      return qc::fail(QCONV_ERR_CUDA, "%s failed: %s", #expr, cudaGetErrorString(e_));        \
  } while (0)

// Device memory of the handles' tables and scratch.  A network's calibration builds and destroys two handles per layer;
// cudaMalloc and cudaFree took two thirds of that time, and at times a hundred milliseconds for one call.  Blocks given back are kept for the next handle, at most kKeep bytes per
// device, and all of them are freed when the last block in use is given back, or when the device has no memory left.  Any thread, any stream: a block is only
// given back after the device is idle, so whoever takes it next may overwrite it at once.
class DevicePool {
 public:
  struct Block {
    void* ptr = nullptr;
    size_t bytes = 0;
    int device = 0;
    Block() = default;
    Block(const Block&) = delete;
    Block& operator=(const Block&) = delete;
    ~Block() { if (ptr) pool().give(*this); }
  };
  static DevicePool& pool() {
    static DevicePool* p = new DevicePool;                 // never destroyed: handles may outlive static destructors
    return *p;
  }
  cudaError_t take(Block* b, size_t bytes) {
    bytes = (std::max<size_t>(bytes, 1) + 4095) / 4096 * 4096;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    b->device = dev;
    std::lock_guard<std::mutex> lock(mu_);
    PerDevice& d = per_device_[dev & 63];
    size_t best = d.free.size();
    for (size_t i = 0; i < d.free.size(); ++i)
      if (d.free[i].second >= bytes && d.free[i].second <= 2 * bytes && (best == d.free.size() || d.free[i].second < d.free[best].second))
        best = i;
    if (best < d.free.size()) {
      b->ptr = d.free[best].first;
      b->bytes = d.free[best].second;
      d.kept -= b->bytes;
      d.free.erase(d.free.begin() + static_cast<long>(best));
    } else {
      e = allocate(&b->ptr, bytes, d);
      if (e != cudaSuccess) { b->ptr = nullptr; return e; }
      b->bytes = bytes;
    }
    ++d.live;
    return cudaSuccess;
  }
  // cudaMalloc for memory that is not the pool's.
  template <typename T>
  cudaError_t plain(T** ptr, size_t bytes) {
    int dev = 0;
    const cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    std::lock_guard<std::mutex> lock(mu_);
    return allocate(reinterpret_cast<void**>(ptr), bytes, per_device_[dev & 63]);
  }

 private:
  static constexpr size_t kKeep = 256u << 20;
  struct PerDevice {
    std::vector<std::pair<void*, size_t>> free;            // oldest first
    size_t kept = 0, live = 0;
  };
  std::mutex mu_;
  PerDevice per_device_[64];

  // On a full device what is kept for later handles goes first.  (Kept blocks are idle.)
  cudaError_t allocate(void** ptr, size_t bytes, PerDevice& d) {
    cudaError_t e = cudaMalloc(ptr, bytes);
    if (e != cudaErrorMemoryAllocation || d.free.empty()) return e;
    cudaGetLastError();
    for (auto& f : d.free) cudaFree(f.first);
    d.free.clear();
    d.kept = 0;
    return cudaMalloc(ptr, bytes);
  }
  void give(Block& b) {
    int dev = 0;
    const bool other = cudaGetDevice(&dev) == cudaSuccess && dev != b.device && cudaSetDevice(b.device) == cudaSuccess;
    const bool idle = cudaDeviceSynchronize() == cudaSuccess;
    std::vector<void*> drop;
    {
      std::lock_guard<std::mutex> lock(mu_);
      PerDevice& d = per_device_[b.device & 63];
      --d.live;
      if (idle) { d.free.emplace_back(b.ptr, b.bytes); d.kept += b.bytes; } else { drop.push_back(b.ptr); }
      size_t n = 0;
      while (n < d.free.size() && (d.live == 0 || d.kept > kKeep)) { drop.push_back(d.free[n].first); d.kept -= d.free[n].second; ++n; }
      d.free.erase(d.free.begin(), d.free.begin() + static_cast<long>(n));
    }
    for (void* p : drop) cudaFree(p);
    if (other) cudaSetDevice(dev);
    b.ptr = nullptr;
  }
};
