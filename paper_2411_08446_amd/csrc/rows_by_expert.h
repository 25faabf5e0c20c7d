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
  int expert;           // -1: there is no such tile
  int64_t first, end;   // its first row, the end of its expert's rows
  int column;           // its tile of columns
};

// The experts' row tiles of `tile` rows, in the order of the experts.  Every wave counts them by itself: lane e % 64 has expert
// e's, summed over the lanes.  The first 64 experts' counts stay in registers.
struct RowTiles {
  const int32_t* offsets;
  int64_t rows;
  int E, tile;
  int lo, hi, upto;     // of expert `lane`: its rows, the tiles up to and with it
  int64_t total;

  __device__ __forceinline__ void count(int e0, int& lo_, int& hi_, int& upto_) const {
    const int lane = (int)threadIdx.x % kWave;
    RowRange range = {0, 0};
    if (e0 + lane < E) range = rows_of(offsets, e0 + lane, rows);
    lo_ = (int)range.lo;
    hi_ = (int)range.hi;
    upto_ = (hi_ - lo_ + tile - 1) / tile;
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) {
      const int below = __shfl_up(upto_, s, kWave);
      if (lane >= s) upto_ += below;
    }
  }

  __device__ __forceinline__ RowTiles(const int32_t* __restrict__ offsets_, int E_, int64_t rows_, int tile_)
      : offsets(offsets_), rows(rows_), E(E_), tile(tile_) {
    count(0, lo, hi, upto);
    total = __builtin_amdgcn_readlane(upto, kWave - 1);
    for (int e0 = kWave; e0 < E; e0 += kWave) {
      int l, h, u;
      count(e0, l, h, u);
      total += __builtin_amdgcn_readlane(u, kWave - 1);
    }
  }

  // Tile n of the experts' row tiles by `columns` tiles of columns.  An expert's tiles go in bands of kBand row tiles, within a
  // band column after column: the tiles that run at a time on an XCD are about as many rows as columns wide and share
  // what they read.
  __device__ __forceinline__ RowTile find(int64_t n, int columns) const {
    constexpr int kBand = 4;
    const int64_t m = n / columns;
    int64_t before = 0;                       // tiles of the experts below e0
    int l = lo, h = hi, u = upto;
    for (int e0 = 0;;) {
      const uint64_t past = __ballot(before + u > m);
      if (past != 0) {
        const int at = __ffsll((unsigned long long)past) - 1;
        const int rlo = __builtin_amdgcn_readlane(l, at), rhi = __builtin_amdgcn_readlane(h, at);
        const int count_at = (rhi - rlo + tile - 1) / tile;
        const int64_t inside = n - (before + __builtin_amdgcn_readlane(u, at) - count_at) * columns;   // its number in the expert
        const int band = (int)(inside / ((int64_t)kBand * columns)), rest = (int)(inside - (int64_t)band * kBand * columns);
        const int wide = min(kBand, count_at - band * kBand);
        return {e0 + at, rlo + (int64_t)(band * kBand + rest % wide) * tile, rhi, rest / wide};
      }
      before += __builtin_amdgcn_readlane(u, kWave - 1);
      e0 += kWave;
      if (e0 >= E) return {-1, 0, 0, 0};
      count(e0, l, h, u);
    }
  }
};

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
