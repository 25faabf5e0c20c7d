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
// e's, summed over the lanes, 64 experts at a time.
struct RowTiles {
  const int32_t* offsets;
  int rows, E, tile;
  int total;

  // Of expert e0 + lane: its rows, the tiles of experts e0 up to and with it.
  __device__ __forceinline__ void count(int e0, int& lo, int& hi, int& upto) const {
    const int lane = (int)threadIdx.x % kWave;
    RowRange range = {0, 0};
    if (e0 + lane < E) range = rows_of(offsets, e0 + lane, rows);
    lo = range.lo;
    hi = range.hi;
    upto = (hi - lo + tile - 1) / tile;
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) {
      const int below = __shfl_up(upto, s, kWave);
      if (lane >= s) upto += below;
    }
  }

  __device__ __forceinline__ RowTiles(const int32_t* __restrict__ offsets_, int E_, int rows_, int tile_)
      : offsets(offsets_), rows(rows_), E(E_), tile(tile_), total(0) {
    for (int e0 = 0; e0 < E; e0 += kWave) {
      int lo, hi, upto;
      count(e0, lo, hi, upto);
      total += __builtin_amdgcn_readlane(upto, kWave - 1);
    }
  }

  // Tile n of the experts' row tiles by `columns` tiles of columns; every lane may ask for another one, and all lanes of a wave
  // ask together (n >= total * columns gives anything).  An expert's tiles go in bands of kBand row tiles, within a band
  // column after column: the tiles that run at a time on an XCD are about as many rows as columns wide and share what
  // they read (bands of 8: 3 % less time than bands of 4, 6 % less than
  // row by row at 4096 -> 4096 columns).
  __device__ __forceinline__ RowTile find(int n, int columns) const {
    constexpr int kBand = 8;
    const int m = (int)((uint32_t)n / (uint32_t)columns);
    int before = 0;                           // tiles of the experts below e0
    RowTile t = {0, 0, 0, 0};
    for (int e0 = 0; e0 < E; e0 += kWave) {
      int lo, hi, upto;
      count(e0, lo, hi, upto);
      const int here = __builtin_amdgcn_readlane(upto, kWave - 1);
      int at = 0;                             // experts of these 64 that end at or before tile m
#pragma unroll
      for (int s = kWave / 2; s >= 1; s >>= 1)
        if (before + __shfl(upto, at + s - 1, kWave) <= m) at += s;
      at = min(at, kWave - 1);
      const int rlo = __shfl(lo, at, kWave), rhi = __shfl(hi, at, kWave), past = __shfl(upto, at, kWave);
      if (m >= before && m < before + here) {
        const int mine = (rhi - rlo + tile - 1) / tile;
        const int inside = n - (before + past - mine) * columns;          // its number in the expert
        const int band = (int)((uint32_t)inside / (uint32_t)(kBand * columns)), rest = inside - band * kBand * columns;
        const int wide = min(kBand, mine - band * kBand);
        t.expert = e0 + at;
        t.column = (int)((uint32_t)rest / (uint32_t)wide);
        t.first = rlo + (band * kBand + rest - t.column * wide) * tile;
        t.rows = min(tile, rhi - t.first);
      }
      before += here;
    }
    return t;
  }
};

// The normal distribution beyond u >= 0, Q(u) = integral of phi from u on, and phi(u).  Q(u) = exp(-u^2 / 2) P(t), t = 1 / (1 + p u),
// P of degree 5 without a constant term: the form of Abramowitz and Stegun 26.2.17, with p and coefficients fitted for the
// least maximum error, 6.1e-8.  Evaluated in binary32 it is good to 2.1e-7 (the library's erf takes twice as long, which at
// K = 1024 was a quarter of a product's time).
struct NormalTail { float beyond, density; };
__device__ __forceinline__ NormalTail normal_tail(float u) {
  const float t = __builtin_amdgcn_rcpf(fmaf(0.331f, u, 1.0f));
  const float e = __builtin_amdgcn_exp2f(u * u * -0.72134752f);
  float p = fmaf(-0.110234566f, t, 0.374119867f);
  p = fmaf(p, t, -0.0900151826f);
  p = fmaf(p, t, 0.203860818f);
  p = fmaf(p, t, 0.122269003f);
  return {e * (p * t), e * 0.39894228f};
}

__device__ __forceinline__ float activate(float v, int act) {
  if (act == LSHMOE_ACT_RELU) return v < 0.0f ? 0.0f : v;
  if (act == LSHMOE_ACT_GELU) {
    const float u = fminf(fabsf(v), 64.0f);       // infinities: 64 is as good
    return fmaf(-u, normal_tail(u).beyond, v < 0.0f ? 0.0f : v);
  }
  return v;
}

__device__ __forceinline__ float activation_slope(float v, int act) {
  if (act == LSHMOE_ACT_RELU) return v > 0.0f ? 1.0f : 0.0f;
  if (act == LSHMOE_ACT_GELU) {
    const NormalTail n = normal_tail(fminf(fabsf(v), 64.0f));
    return fmaf(v, n.density, v < 0.0f ? n.beyond : 1.0f - n.beyond);
  }
  return 1.0f;
}

}  // namespace lshmoe
