// Shared memory that a launch in clusters asks for beside its tensor memory; plain C++.
//
// tcgen05.alloc waits until its columns are free, and the barriers of a cluster wait for all of its CTAs; neither wait can be
// bounded.  CTAs are placed by shared memory, registers and threads alone: the columns are not counted.  If
// clusters of two streams met on SMs whose columns do not suffice for both, each could hold columns on one SM while its other
// CTA waits for the other's on the next, for ever.  So every cluster's CTA asks for at least its columns' part of an SM's shared
// memory: clusters' CTAs that fit an SM by their shared memory then fit by their columns, and none of them waits for another's.
// (CTAs outside of clusters need no such part: they hold columns only while they run, and give them back in bounded time.  Nor do
// kernels of one stream: each starts the next only once all of its CTAs have their columns.)
#pragma once
#include <cstddef>

namespace qc {

constexpr size_t kSmSharedBytes = 228 * 1024, kCtaReservedBytes = 1024;   // of an SM; the system's part of each CTA's
constexpr int kSmTmemColumns = 512;

// Dynamic shared memory of a cluster's CTA that needs `needed` bytes and allocates `columns` columns.
constexpr size_t cluster_smem(size_t needed, int columns) {
  const size_t part = static_cast<size_t>(columns) * (kSmSharedBytes / kSmTmemColumns) - kCtaReservedBytes;
  return needed > part ? needed : part;
}
static_assert(kSmSharedBytes % kSmTmemColumns == 0 && cluster_smem(0, kSmTmemColumns) == 227 * 1024);   // what a CTA can ask for

}  // namespace qc
