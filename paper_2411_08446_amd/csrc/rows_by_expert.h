// Rows grouped by expert, as the experts' products see them: which expert and which rows a workgroup has, from offsets in
// device memory, and the activations.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

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

// Things of the experts (row tiles, parts of their rows), numbered in the order of the experts; pieces(n) says how many an expert
// of n rows has.  Every wave counts them by itself: lane e % 64 has expert e's, summed over the lanes, 64 experts at a time.
template <typename PIECES> struct ByExpert {
  const int32_t* offsets;
  int rows, E;
  PIECES pieces;
  int total;
  RowRange range0;        // what count(0, ..) gives
  int mine0, upto0;

  // Of expert e0 + lane: its rows, how many it has, how many experts e0 up to and with it have.  AGAIN: not from what is kept, which
  // would stay in registers until then.
  template <bool AGAIN = false>
  __device__ __forceinline__ void count(int e0, RowRange& range, int& mine, int& upto) const {
    if (!AGAIN && e0 == 0) {
      range = range0;
      mine = mine0;
      upto = upto0;
    } else {
      look(e0, range, mine, upto);
    }
  }
  __device__ __forceinline__ void look(int e0, RowRange& range, int& mine, int& upto) const {
    const int lane = (int)threadIdx.x % kWave;
    range = {0, 0};
    mine = 0;
    if (e0 + lane < E) {
      range = rows_of(offsets, e0 + lane, rows);
      mine = pieces(range.hi - range.lo);
    }
    upto = mine;
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) {
      const int below = __shfl_up(upto, s, kWave);
      if (lane >= s) upto += below;
    }
  }

  __device__ __forceinline__ ByExpert(const int32_t* __restrict__ offsets_, int E_, int rows_, const PIECES& pieces_)
      : offsets(offsets_), rows(rows_), E(E_), pieces(pieces_), total(0) {
    look(0, range0, mine0, upto0);
    total = __builtin_amdgcn_readlane(upto0, kWave - 1);
    for (int e0 = kWave; e0 < E; e0 += kWave) {
      RowRange range;
      int mine, upto;
      count(e0, range, mine, upto);
      total += __builtin_amdgcn_readlane(upto, kWave - 1);
    }
  }

  struct Found {
    int expert;
    RowRange range;
    int count, number;    // how many its expert has, which of them it is
  };
  // Number m; every lane may ask for another one, and all lanes of a wave ask together (m >= total gives expert 0 with
  // nothing).
  template <bool AGAIN = false> __device__ __forceinline__ Found find(int m) const {
    int before = 0;                           // of the experts below e0
    Found f = {0, {0, 0}, 0, 0};
    for (int e0 = 0; e0 < E; e0 += kWave) {
      RowRange range;
      int mine, upto;
      count<AGAIN>(e0, range, mine, upto);
      const int here = __builtin_amdgcn_readlane(upto, kWave - 1);
      int at = 0;                             // experts of these 64 that end at or before m
#pragma unroll
      for (int s = kWave / 2; s >= 1; s >>= 1)
        if (before + __shfl(upto, at + s - 1, kWave) <= m) at += s;
      at = min(at, kWave - 1);
      const RowRange there = {__shfl(range.lo, at, kWave), __shfl(range.hi, at, kWave)};
      const int past = __shfl(upto, at, kWave), its = __shfl(mine, at, kWave);
      if (m >= before && m < before + here) f = {e0 + at, there, its, m - (before + past - its)};
      before += here;
    }
    return f;
  }
};

struct TilePieces {
  int tile;
  __device__ __forceinline__ int operator()(int n) const { return (n + tile - 1) / tile; }
};

// The experts' row tiles of `tile` rows.
struct RowTiles : ByExpert<TilePieces> {
  __device__ __forceinline__ RowTiles(const int32_t* __restrict__ offsets_, int E_, int rows_, int tile_)
      : ByExpert(offsets_, E_, rows_, TilePieces{tile_}) {}

  // Tile n of the experts' row tiles by `columns` tiles of columns; lanes as above.  An expert's tiles go in bands of kBand row
  // tiles, within a band column after column: the tiles that run at a time on an XCD are about as many rows as columns
  // wide and share what they read (bands of 8: 3 % less time than bands of 4, 6 % less than row by row at 4096 -> 4096
  // columns).
  template <bool AGAIN = false> __device__ __forceinline__ RowTile tile(int n, int columns) const {
    constexpr int kBand = 8;
    const int m = (int)((uint32_t)n / (uint32_t)columns);
    const Found f = find<AGAIN>(m);
    const int inside = f.number * columns + (n - m * columns);            // its number in the expert
    const int band = (int)((uint32_t)inside / (uint32_t)(kBand * columns)), rest = inside - band * kBand * columns;
    const int wide = max(min(kBand, f.count - band * kBand), 1);
    RowTile t;
    t.expert = f.expert;
    t.column = (int)((uint32_t)rest / (uint32_t)wide);
    t.first = f.range.lo + (band * kBand + rest - t.column * wide) * pieces.tile;
    t.rows = min(pieces.tile, f.range.hi - t.first);
    return t;
  }
};

// Parts of at most `goal` rows and a twentieth for the sums over an expert's rows; an expert without rows is one part.  Part k of
// `count` of n rows begins at k n / count, the next one more than goal / 2 rows behind it.
struct RowPieces {
  int goal;
  __device__ __forceinline__ int operator()(int n) const {
    return max((int)((uint32_t)(n + (goal - goal / 64 * 3)) / (uint32_t)goal), 1);
  }
};
__device__ __forceinline__ int part_start(const RowRange& range, int count, int k) {
  return range.lo + (int)((int64_t)(range.hi - range.lo) * k / max(count, 1));
}

struct RowParts : ByExpert<RowPieces> {
  __device__ __forceinline__ RowParts(const int32_t* __restrict__ offsets_, int E_, int rows_, int goal)
      : ByExpert(offsets_, E_, rows_, RowPieces{goal}) {}

  // All parts' tiles, `tiles` to a part, in `of` runs of about the same work: where run x begins and ends.  A tile's work is its rows
  // and kOver more for what does not depend on them.
  __device__ __forceinline__ RowRange run_of_work(int x, int of, int tiles) const {
    constexpr int kOver = 256;
    const int64_t whole = (int64_t)rows_of(offsets, E - 1, rows).hi + (int64_t)kOver * total;
    int before = 0, n[2] = {0, 0};
    for (int e0 = 0; e0 < E; e0 += kWave) {
      RowRange range;
      int mine, upto;
      count(e0, range, mine, upto);
      const int64_t start = range.lo + (int64_t)kOver * (before + upto - mine);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int64_t goal = whole * (x + i) / of;
        const uint64_t begun = __ballot(mine > 0 && start <= goal);
        if (begun == 0) continue;
        const int at = kWave - 1 - __builtin_clzll(begun);        // the last expert that begins at or before the goal
        const RowRange r = {__builtin_amdgcn_readlane(range.lo, at), __builtin_amdgcn_readlane(range.hi, at)};
        const int its = __builtin_amdgcn_readlane(mine, at), first = before + __builtin_amdgcn_readlane(upto, at) - its;
        const int64_t into = goal - (r.lo + (int64_t)kOver * first), each = (r.hi - r.lo) / its + kOver;
        const int k = (int)min(into / each, (int64_t)its - 1);
        n[i] = (first + k) * tiles + (int)min((into - k * each) * tiles / each, (int64_t)tiles);
      }
      before += __builtin_amdgcn_readlane(upto, kWave - 1);
    }
    const int all = total * tiles;
    return {x == 0 ? 0 : min(n[0], all), x + 1 == of ? all : min(n[1], all)};
  }
};

// The normal distribution beyond u >= 0, Q(u) = integral of phi from u on, and phi(u).  Q(u) = exp(-u^2 / 2) P(t), t = 1 / (1 + p u),
// P a polynomial without a constant term: the form of Abramowitz and Stegun 26.2.17, with p and coefficients fitted.  What is
// wanted is a small error relative to Q, since v Phi(v) is -u Q(u) for v = -u: one that is small beside 1 leaves few bits of
// the far tail.
//   bf16 results: degree 6, off by at most 2^-11 of Q (an eighth of the result's half step) and 2e-7.
//   binary32 results: degree 10, 7e-9 of Q; with it the exponent of the exponential is held in two numbers (u^2 reaches 170, and its
//   rounding counts as often in the result): within 20 units of 2^-24 of Q, mostly within 2.
// The library's erf takes twice as long as the first, which at K = 1024 was a quarter of a product's time.  Below 2^-126 is 0.
struct NormalTail { float beyond, density; };
template <typename DT> __device__ __forceinline__ NormalTail normal_tail(float u) {
  constexpr float kHalfLog2e = -0.72134752f, kDensity0 = 0.39894228f;
  const float square = u * u;
  if constexpr (std::is_same<DT, F32>::value) {
    constexpr float kHalfLog2eRest = -9.62981517e-9f, kLn2 = 0.69314718f;
    const float t = __builtin_amdgcn_rcpf(fmaf(0.385f, u, 1.0f));
    const float x = square * kHalfLog2e;
    float rest = fmaf(square, kHalfLog2e, -x);
    rest = fmaf(fmaf(u, u, -square), kHalfLog2e, rest);
    rest = fmaf(square, kHalfLog2eRest, rest);
    float e = __builtin_amdgcn_exp2f(x);
    e = fmaf(e * kLn2, rest, e);
    float p = fmaf(0.0269641951f, t, -0.160244823f);
    p = fmaf(p, t, 0.38198477f);
    p = fmaf(p, t, -0.431546152f);
    p = fmaf(p, t, 0.195146635f);
    p = fmaf(p, t, -0.0513688661f);
    p = fmaf(p, t, 0.103469275f);
    p = fmaf(p, t, 0.128202856f);
    p = fmaf(p, t, 0.153806835f);
    p = fmaf(p, t, 0.153585255f);
    return {e * (p * t), e * kDensity0};
  } else {
    const float t = __builtin_amdgcn_rcpf(fmaf(0.41f, u, 1.0f));
    const float e = __builtin_amdgcn_exp2f(square * kHalfLog2e);
    float p = fmaf(0.0555896088f, t, -0.238357916f);
    p = fmaf(p, t, 0.287518591f);
    p = fmaf(p, t, 0.0531319417f);
    p = fmaf(p, t, 0.179703563f);
    p = fmaf(p, t, 0.162414268f);
    return {e * (p * t), e * kDensity0};
  }
}

// DT: type of the result.
template <typename DT> __device__ __forceinline__ float activate(float v, int act) {
  const float above = __builtin_elementwise_maximum(v, 0.0f);     // one instruction, a NaN stays one
  if (act == LSHMOE_ACT_RELU) return above;
  if (act == LSHMOE_ACT_GELU) {
    const float u = fminf(fabsf(v), 64.0f);       // infinities: 64 is as good
    return fmaf(-u, normal_tail<DT>(u).beyond, above);
  }
  return v;
}

template <typename DT> __device__ __forceinline__ float activation_slope(float v, int act) {
  if (act == LSHMOE_ACT_RELU) return v > 0.0f ? 1.0f : 0.0f;
  if (act == LSHMOE_ACT_GELU) {
    const float u = fabsf(v) > 64.0f ? 64.0f : fabsf(v);        // as above; a NaN stays one
    const NormalTail n = normal_tail<DT>(u);
    return fmaf(copysignf(u, v), n.density, v < 0.0f ? n.beyond : 1.0f - n.beyond);
  }
  return 1.0f;
}

}  // namespace lshmoe
