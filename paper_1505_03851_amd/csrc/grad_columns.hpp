// The columns of a gradient's rows among the lanes of a wavefront.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lda {

// Tiles of 64 W columns, one to a wavefront, that cover D.
template <int W>
constexpr uint32_t column_tiles(int64_t D) {
  return (uint32_t)((D + 64 * W - 1) / (64 * W));
}

// A lane's columns: n of the W from `own` on exist; it reads, without a branch,
// the W columns from `col` on, which end where they do (in the last lanes some are
// the lane's before).  D is at least W and below 2^31, so `own` passes 31 bits in
// the last tile, and a row is longer than 32-bit byte offsets reach: reads start at
// `first`, which is the same for the wavefront, and a lane's lie `offset` elements
// from there, fewer than 64 W.
template <int W>
struct Columns {
  uint32_t own;
  int32_t n, col, first;
  uint32_t offset;
  __device__ __forceinline__ Columns(uint32_t tile, int32_t D) {
    const uint32_t end = (uint32_t)D, last = end - W, start = tile * (64 * W);
    own = start + (threadIdx.x & 63) * W;
    n = own < end ? (end - own < W ? (int32_t)(end - own) : W) : 0;
    col = (int32_t)(own < last ? own : last);
    first = (int32_t)(start < last ? start : last);
    offset = (uint32_t)(col - first);
  }
};

}  // namespace lda
