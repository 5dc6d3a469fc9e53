// Where a tensor lies, for the checked build's tests of accesses; plain C++.
#pragma once
#include <cstddef>
#include <cstdint>

#include "any_side.cuh"

namespace qc {

struct Extent {
  uintptr_t lo;
  size_t bytes;
  template <typename T> QC_ANY_SIDE static Extent of(const T* p, size_t count) { return {reinterpret_cast<uintptr_t>(p), count * sizeof(T)}; }
  // Whether the `count` bytes from p on are all the tensor's.
  QC_ANY_SIDE bool has(const void* p, size_t count) const {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p) - lo;       // (below the tensor: larger than any extent)
    return at < bytes && count <= bytes - at;
  }
};

}  // namespace qc
