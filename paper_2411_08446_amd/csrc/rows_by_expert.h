// Rows grouped by expert, as the experts' products see them: which expert and which rows a workgroup has, from offsets in
// device memory, and the activations.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/lshmoe.h"
#include "common.h"

namespace lshmoe {

struct RowRange { int lo, hi; };

// Rows of expert e.  Offsets are the caller's: whatever they are, the rows lie in 0 .. rows.
__device__ __forceinline__ RowRange rows_of(const int32_t* __restrict__ offsets, int e, int rows) {
  const int lo = min(max(offsets[e], 0), rows);
  return {lo, min(max(offsets[e + 1], lo), rows)};
}

// Row tiles of `tile` rows that all experts together can have: an expert's last one may be partly empty.
inline int64_t most_row_tiles(int64_t rows, int E, int tile) { return rows / tile + (E < rows ? E : rows); }

struct RowTile {
  int expert;
  int first, rows;      // its first row, how many there are from there to the end of its expert's rows (at most `tile`)
  int column;           // its tile of columns
};

// The experts' row tiles of `tile` rows, in the order of the experts.  Every wave counts them by itself: lane e % 64 has expert
// e's, summed over the lanes.  The first 64 experts' counts stay in registers.
struct RowTiles {
  const int32_t* offsets;
  int rows, E, tile;
  int lo, hi, upto;     // of expert `lane`: its rows, the tiles up to and with it
  int total;

  __device__ __forceinline__ void count(int e0, int& lo_, int& hi_, int& upto_) const {
    const int lane = (int)threadIdx.x % kWave;
    RowRange range = {0, 0};
    if (e0 + lane < E) range = rows_of(offsets, e0 + lane, rows);
    lo_ = range.lo;
    hi_ = range.hi;
    upto_ = (hi_ - lo_ + tile - 1) / tile;
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) {
      const int below = __shfl_up(upto_, s, kWave);
      if (lane >= s) upto_ += below;
    }
  }

  __device__ __forceinline__ RowTiles(const int32_t* __restrict__ offsets_, int E_, int rows_, int tile_)
      : offsets(offsets_), rows(rows_), E(E_), tile(tile_) {
    count(0, lo, hi, upto);
    total = __builtin_amdgcn_readlane(upto, kWave - 1);
    for (int e0 = kWave; e0 < E; e0 += kWave) {
      int l, h, u;
      count(e0, l, h, u);
      total += __builtin_amdgcn_readlane(u, kWave - 1);
    }
  }

  // Rows of expert e.
  __device__ __forceinline__ RowRange range(int e) const {
    if (e < kWave) return {__builtin_amdgcn_readlane(lo, e), __builtin_amdgcn_readlane(hi, e)};
    const RowRange r = rows_of(offsets, e, rows);
    return {__builtin_amdgcn_readfirstlane(r.lo), __builtin_amdgcn_readfirstlane(r.hi)};
  }

  // Tile n < total * columns of the experts' row tiles by `columns` tiles of columns.  An expert's tiles go in bands of kBand row
  // tiles, within a band column after column: the tiles that run at a time on an XCD are about as many rows as columns
  // wide and share what they read (bands of 4: 3 % less time than row by row at 4096 -> 4096 columns).
  __device__ __forceinline__ RowTile find(int n, int columns) const {
    constexpr int kBand = 4;
    const int m = (int)((uint32_t)n / (uint32_t)columns);
    int before = 0;                           // tiles of the experts below e0
    int l = lo, h = hi, u = upto;
    for (int e0 = 0;;) {
      const uint64_t past = __ballot(before + u > m);
      if (past != 0) {
        const int at = __ffsll((unsigned long long)past) - 1;
        const int rlo = __builtin_amdgcn_readlane(l, at), rhi = __builtin_amdgcn_readlane(h, at);
        const int mine = (rhi - rlo + tile - 1) / tile;
        const int inside = n - (before + __builtin_amdgcn_readlane(u, at) - mine) * columns;   // its number in the expert
        const int band = (int)((uint32_t)inside / (uint32_t)(kBand * columns)), rest = inside - band * kBand * columns;
        const int wide = min(kBand, mine - band * kBand);
        const int column = (int)((uint32_t)rest / (uint32_t)wide), first = rlo + (band * kBand + rest - column * wide) * tile;
        return {e0 + at, first, min(tile, rhi - first), column};
      }
      before += __builtin_amdgcn_readlane(u, kWave - 1);
      e0 += kWave;
      if (e0 >= E) return {0, 0, 0, 0};       // not reached for n < total * columns
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
