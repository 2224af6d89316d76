// How the eviction cuts the rows of a long cache: plain arithmetic, which the host
// and the kernels share and a test checks without a GPU. Row numbers are 32 bits; no
// sum here passes them for any length up to kMostRows.
#pragma once

#include <cstdint>

namespace radar_impl {

constexpr int kSelThreads = 1024, kPer = 8;
constexpr int kStep = kSelThreads * kPer;  // rows that a workgroup takes at a time
constexpr int kSlices = 32;                // at most
constexpr int64_t kMostRows = INT32_MAX - 2 * kStep;   // row numbers of a step fit 32 bits

// rows of a slice: whole steps, and at most kSlices slices of t rows
constexpr int64_t slice_rows_of(int64_t t) {
  const int64_t steps = (t + kStep - 1) / kStep;
  return (steps + kSlices - 1) / kSlices * kStep;
}
// the slices that hold rows of a sequence of len > 0 (len + slice_rows may pass 2^31)
constexpr int slices_of(int len, int slice_rows) { return (len - 1) / slice_rows + 1; }
// the end of the slice that begins at `begin` (which may lie behind len)
constexpr int slice_end(int len, int begin, int slice_rows) {
  return len - begin < slice_rows ? len : begin + slice_rows;
}

// What moves a head's rows is launched as one workgroup of kMoveThreads for each
// kMoveBytes of K and of V, and a launch has fewer than 2^32 threads along x.
constexpr int kMoveThreads = 1024, kMoveVecs = 8;
constexpr int kMoveBytes = kMoveThreads * kMoveVecs * 16;
constexpr int64_t move_chunks(int64_t rows, int row_bytes) {
  return (rows * row_bytes + kMoveBytes - 1) / kMoveBytes;
}
constexpr int64_t kMostChunks = (((int64_t)1 << 32) - 1) / kMoveThreads;

}  // namespace radar_impl
