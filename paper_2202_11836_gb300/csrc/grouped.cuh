// Which group a tile of a ragged matrix belongs to (device code).
#pragma once
#include "common.cuh"

namespace sky {
namespace grouped {

// The rows of group g, inside [0, rows] whatever the offsets hold.
__device__ __forceinline__ int2 group_rows(const int32_t* offset, int g, int rows) {
  const int lo = min(max(offset[g], 0), rows);
  return make_int2(lo, min(max(offset[g + 1], lo), rows));
}

struct Found {
  int group;   // -1: there are no so many tiles
  int lo, hi;  // its rows
  int tile;    // of the group's tiles
};

// The tile-th of all groups' tiles, tiles_of(n) of a group of n rows: a whole warp, 32 groups
// at a time.
template <typename F>
__device__ __forceinline__ Found find_tile(const int32_t* offset, int groups, int rows, int tile, F&& tiles_of) {
  const int lane = threadIdx.x & 31;
  for (int g0 = 0; g0 < groups; g0 += 32) {
    int2 r = make_int2(0, 0);
    if (g0 + lane < groups) r = group_rows(offset, g0 + lane, rows);
    const int n = tiles_of(r.y - r.x);
    int upto = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += up;
    }
    const uint32_t past = __ballot_sync(0xffffffffu, tile < upto);
    if (past) {
      const int at = __ffs(past) - 1;
      return {g0 + at, __shfl_sync(0xffffffffu, r.x, at), __shfl_sync(0xffffffffu, r.y, at),
              tile - __shfl_sync(0xffffffffu, upto - n, at)};
    }
    tile -= __shfl_sync(0xffffffffu, upto, 31);
  }
  return {-1, 0, 0, 0};
}

// Sets the bad-length bit where the offsets decrease or leave [0, rows]: by one thread block.
__device__ __forceinline__ void check_offsets(const int32_t* offset, int groups, int rows, int32_t* status) {
  if (!status) return;
  for (int g = threadIdx.x; g < groups; g += blockDim.x)
    if (offset[g] < 0 || offset[g + 1] < offset[g] || offset[g + 1] > rows) atomicOr(status, kStatusBadLength);
}

}  // namespace grouped
}  // namespace sky
