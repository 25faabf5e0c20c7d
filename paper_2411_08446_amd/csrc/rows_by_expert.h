// Rows grouped by expert, as the experts' products see them: which expert and which rows a workgroup has, from offsets in
// device memory, and the activations.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/lshmoe.h"
#include "common.h"

namespace lshmoe {

struct RowRange { int64_t lo, hi; };

// Rows of expert e.  Offsets are the caller's: whatever they are, the rows lie in 0 .. rows.
__device__ __forceinline__ RowRange rows_of(const int32_t* __restrict__ offsets, int e, int64_t rows) {
  const int lo = min(max(offsets[e], 0), (int)rows);
  return {lo, min(max(offsets[e + 1], lo), (int)rows)};
}

// Row tiles of `tile` rows that all experts together can have: an expert's last one may be partly empty.
inline int64_t most_row_tiles(int64_t rows, int E, int tile) { return rows / tile + (E < rows ? E : rows); }

struct RowTile {
  int expert;           // -1: there are fewer row tiles than that
  int64_t first, end;   // its first row, the end of its expert's rows
};

// Row tile number m of all experts' row tiles, in the order of the experts.  Every wave finds it by itself: lane e % 64 counts
// expert e's tiles and the counts are summed over the lanes.
__device__ __forceinline__ RowTile find_row_tile(const int32_t* __restrict__ offsets, int E, int64_t rows, int tile, int64_t m) {
  const int lane = (int)threadIdx.x % kWave;
  int64_t before = 0;                         // tiles of the experts below e0
  for (int e0 = 0; e0 < E; e0 += kWave) {
    RowRange range = {0, 0};
    if (e0 + lane < E) range = rows_of(offsets, e0 + lane, rows);
    const int tiles = (int)((range.hi - range.lo + tile - 1) / tile);
    int upto = tiles;
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) {
      const int below = __shfl_up(upto, s, kWave);
      if (lane >= s) upto += below;
    }
    const uint64_t past = __ballot(before + upto > m);
    if (past != 0) {
      const int at = __ffsll((unsigned long long)past) - 1;
      const int lo = __builtin_amdgcn_readlane((int)range.lo, at), hi = __builtin_amdgcn_readlane((int)range.hi, at);
      const int64_t skipped = m - before - (__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(tiles, at));
      return {e0 + at, lo + skipped * tile, hi};
    }
    before += __builtin_amdgcn_readlane(upto, kWave - 1);
  }
  return {-1, 0, 0};
}

__device__ __forceinline__ float activate(float v, int act) {
  if (act == LSHMOE_ACT_RELU) return v > 0.0f || v != v ? v : 0.0f;
  if (act == LSHMOE_ACT_GELU) return 0.5f * v * (1.0f + erff(v * 0.70710678f));
  return v;
}

__device__ __forceinline__ float activation_slope(float v, int act) {
  if (act == LSHMOE_ACT_RELU) return v > 0.0f ? 1.0f : 0.0f;
  if (act == LSHMOE_ACT_GELU) return 0.5f * (1.0f + erff(v * 0.70710678f)) + v * expf(-0.5f * v * v) * 0.39894228f;
  return 1.0f;
}

}  // namespace lshmoe
