// How the rows of a norm are dealt out to its blocks; plain C++, the host's side and the kernels'.
#pragma once

#include <cstdint>

#ifdef __CUDACC__
#define IRIS_BOTH __host__ __device__ __forceinline__
#else
#define IRIS_BOTH inline
#endif

namespace iris {
namespace rows {

constexpr int kNormPeriod = 8;   // places of 16 bytes where a row may begin

// A group's first row, between rows taken at once, between those and the next ones.  Rows `period` apart begin at the same place of 16 bytes; a block (or
// cluster: `block` of `blocks`) has rows of one such set only, `set`.  index: of the group among the block's; at_once: rows that a group takes at a time.
struct NormWalk {
  int64_t first, each, step;
};
IRIS_BOTH int64_t norm_set(int64_t block, int64_t period) { return block % period; }
IRIS_BOTH NormWalk norm_walk(int64_t block, int64_t blocks, int index, int groups, int64_t period, int64_t set, int at_once) {
  return NormWalk{set + period * (block / period * groups + index) * at_once, period, period * ((blocks - set + period - 1) / period) * groups * at_once};
}
// Blocks (or clusters, of which there are `room` at once): at least one for each place where a row begins, also where fewer fit on the device (they wait for
// none but the blocks of their own cluster).
inline int64_t norm_grid(int groups, int at_once, int64_t rows, int64_t room) {
  const int64_t each = (int64_t)groups * at_once, full = (rows + each - 1) / each, most = rows < kNormPeriod ? rows : kNormPeriod;
  const int64_t fit = full < room ? full : room;
  return fit < most ? most : fit;
}

}  // namespace rows
}  // namespace iris
