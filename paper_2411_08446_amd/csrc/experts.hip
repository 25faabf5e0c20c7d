// The experts' products on rows that are grouped by expert: rows expert_offsets[e] .. expert_offsets[e+1] - 1 belong to
// expert e.  The offsets are in device memory, so a launch is sized for the worst case and a workgroup finds its expert
// and its rows from the offsets itself.
//
//   forward      pre = x W_e^T + b_e,  out = act(pre)          W_e [d_out, d_in]
//   input        grad_x = (grad_out W_e) * act'(pre)
//   weight       grad_W_e = grad_out_e^T x_e,  grad_b_e = sum of grad_out_e
//
// The tiles and how they are computed: product_tile.h.  65536 rows of 64 experts, 1024 -> 4096 columns of bf16: input gradient of
// the second product with the activation's slope 580 us, 0.95 PFLOP/s; weight gradient 508 us, 1.08 PFLOP/s.
#include "kernels.h"
#include "product_direct.h"
#include "product_tile.h"

namespace lshmoe {

namespace {

template <typename DT, typename TILE, int BP, int BQ> struct InputGradJob {
  typedef PlaceOfRows Place;
  static constexpr bool kSums = false;
  static constexpr int kItem = ItemSize<DT>::value;
  const char *grad_out, *w, *pre;
  char* grad_x;
  int d_in, d_out, act, ptiles;
  const RowTiles& tiles;

  __device__ __forceinline__ uint32_t p_stride() const { return (uint32_t)d_in * kItem; }
  __device__ __forceinline__ uint32_t q_stride() const { return (uint32_t)d_out * kItem; }
  __device__ __forceinline__ uint32_t s_stride() const { return 0; }
  template <bool AGAIN> __device__ __forceinline__ TileEntry entry(int n) const {
    const RowTile t = tiles.template tile<AGAIN>(n, ptiles);
    return {{t.expert, t.first, t.rows, t.column * BP, 0}};
  }
  __device__ __forceinline__ Place place(const TileEntry& t) const {
    const int expert = t.v[0], first = t.v[1], nq = t.v[2], p0 = t.v[3];
    return {w + ((int64_t)expert * d_out * d_in + p0) * kItem, grad_out + (int64_t)first * d_out * kItem, nullptr, nullptr,
            min(BP, d_in - p0), nq, d_out, TILE::OpP::kChunk, expert, first, p0};
  }
  __device__ __forceinline__ bool sums(const Place&) const { return false; }
  __device__ __forceinline__ bool twice() const { return false; }
  template <int ACT> __device__ __forceinline__ void store(const Place& at, const TILE& tile) const {
    const int64_t first = ((int64_t)at.first * d_in + at.p0) * kItem;
    const typename TILE::Lines o = TILE::lines(grad_x + first, (uint32_t)d_in * kItem, at.nq, at.np);
    const typename TILE::Lines k = TILE::lines((ACT == LSHMOE_ACT_NONE ? grad_x : pre) + first, (uint32_t)d_in * kItem, at.nq, at.np);
    // The values before the activation come in two halves, both loaded before anything is stored, as in the forward product; the
    // first half's results wait, packed.
    constexpr int kHalf = TILE::kGroups > 1 ? TILE::kGroups / 2 : 1;
    typename TILE::Pieces x[kHalf][TILE::TQ], y[kHalf][TILE::TQ];
    auto get = [&](int g0) {
#pragma unroll
      for (int g = 0; g < kHalf; ++g)
#pragma unroll
        for (int u = 0; u < TILE::TQ; ++u) x[g][u] = TILE::get(k, g0 + g, u);
      asm volatile("" : : : "memory");
    };
    auto scale = [&](int g0) {
#pragma unroll
      for (int g = 0; g < kHalf; ++g)
#pragma unroll
        for (int u = 0; u < TILE::TQ; ++u) {
          constexpr int kElems = 16 * TILE::kGroupTiles;
          float v[kElems];
          tile.results(g0 + g, u, v);
          if (ACT != LSHMOE_ACT_NONE) {
            float z[kElems];
            TILE::spread(x[g][u], z);
#pragma unroll
            for (int i = 0; i < kElems; ++i) v[i] *= activation_slope<DT>(z[i], ACT);
          }
          y[g][u] = TILE::pack(v);
        }
    };
    auto put = [&](int g0) {
#pragma unroll
      for (int g = 0; g < kHalf; ++g)
#pragma unroll
        for (int u = 0; u < TILE::TQ; ++u) TILE::put(o, g0 + g, u, y[g][u]);
    };
    if (ACT != LSHMOE_ACT_NONE) get(0);
    scale(0);
    if constexpr (TILE::kGroups > 1) {
      if (ACT != LSHMOE_ACT_NONE) get(kHalf);
      put(0);
      scale(kHalf);
      put(kHalf);
    } else {
      put(0);
    }
  }
  __device__ __forceinline__ void finish(const Place& at, const TILE& tile) const {
    if (act == LSHMOE_ACT_RELU) store<LSHMOE_ACT_RELU>(at, tile);
    else if (act == LSHMOE_ACT_GELU) store<LSHMOE_ACT_GELU>(at, tile);
    else store<LSHMOE_ACT_NONE>(at, tile);
  }
};

template <typename DT, typename TILE, int BP, int BQ>
__global__ __launch_bounds__(TILE::kThreads, 2) void input_grad_kernel(const char* __restrict__ grad_out,
                                                                       const char* __restrict__ w,
                                                                       const int32_t* __restrict__ offsets, int rows, int d_in,
                                                                       int d_out, int E, int act,
                                                                       const char* __restrict__ pre, char* __restrict__ grad_x) {
  const RowTiles tiles(offsets, E, rows, BQ);
  const int ptiles = (d_in + BP - 1) / BP;
  const InputGradJob<DT, TILE, BP, BQ> job = {grad_out, w, pre, grad_x, d_in, d_out, act, ptiles, tiles};
  const Share s = share_of_block(tiles.total * ptiles);
  TILE tile;
  tile.run(job, s.first, s.end, s.step);
}

// Rows of a part of an expert's rows (see RowParts): a workgroup's share of the work, in binary32 a quarter of that (its products
// take 16 times as long as bf16's, the partial sums' way through memory does not: 576 tiles on 512 workgroups, 15011 rows,
// 1000 -> 1500 columns, 466 -> 402 us).  Parts below 512 rows are not worth that way.
constexpr int kLeastPart = 512;
__host__ __device__ inline int part_rows(int64_t rows, int64_t tiles, int parts) {
  const int64_t share = rows * tiles / parts;
  return (int)(share > kLeastPart ? share : kLeastPart);
}
// Partial sums are kept at the number of their first row over half a part: parts of experts that are cut begin further apart.
inline uint64_t part_slots(int64_t rows, int64_t tiles, int parts) {
  // a share rounded down twice, of 256 rows at least: less than 1 / 64 more slots
  const uint64_t fine = 2 * (uint64_t)parts / (uint64_t)tiles, most = fine + fine / 64 + 2;
  const uint64_t all = (uint64_t)rows / (kLeastPart / 2) + 1;
  return most < all ? most : all;
}

// PARTS: tiles' parts that all workgroups together should have.
template <typename DT> struct WeightGradShape : Large { static constexpr int PARTS = kUnits * kPerUnit; };
template <> struct WeightGradShape<F32> : Small { static constexpr int PARTS = 4 * kUnits * kPerUnit; };

// Gradients of W_e and b_e.  An expert with many rows is cut into parts; a part's sums go to the workspace in binary32, in the
// order in which the lanes hold them, and a second kernel adds the parts up, first to last.
template <typename DT, typename TILE, int BP, int BQ> struct WeightGradJob {
  struct Place {
    const char *p, *q;
    int np, nq, K, expert, p0, q0, tile, slot;    // slot: of the partial sums, or -1: the expert is one part
    __device__ __forceinline__ int chunks() const { return max((K + TILE::OpP::kChunk - 1) / TILE::OpP::kChunk, 1); }
    __device__ __forceinline__ static Place none(const Place& like) {
      Place x = like;
      x.np = x.nq = x.K = 0;
      return x;
    }
  };
  static constexpr bool kSums = true;
  static constexpr int kItem = ItemSize<DT>::value;
  const char *grad_out, *x;
  char *grad_w, *grad_bias;
  float4* partial;        // [slot][tile][TP TQ 4][thread]
  float* partial_sums;    // [slot][tile][TQ][thread]
  int d_in, d_out, ptiles, qtiles, slots;
  const RowParts& parts;

  __device__ __forceinline__ uint32_t p_stride() const { return (uint32_t)d_in * kItem; }
  __device__ __forceinline__ uint32_t q_stride() const { return (uint32_t)d_out * kItem; }
  __device__ __forceinline__ uint32_t s_stride() const { return 0; }
  // (the bound is for offsets that are no offsets)
  __device__ __forceinline__ int slot_of(int first_row) const {
    return min((int)((uint32_t)first_row / (uint32_t)(parts.pieces.goal / 2)), slots - 1);
  }
  template <bool AGAIN> __device__ __forceinline__ TileEntry entry(int n) const {
    const int m = (int)((uint32_t)n / (uint32_t)(ptiles * qtiles));
    return entry_of(parts.template find<AGAIN>(m), n - m * ptiles * qtiles);
  }
  __device__ __forceinline__ TileEntry entry_of(const RowParts::Found& f, int tile) const {
    const int first = part_start(f.range, f.count, f.number), end = part_start(f.range, f.count, f.number + 1);
    return {{f.expert, tile, first, end - first, f.count > 1 ? slot_of(first) : -1}};
  }
  __device__ __forceinline__ Place place(const TileEntry& t) const {
    const int e = t.v[0], q = (int)((uint32_t)t.v[1] / (uint32_t)ptiles), p0 = (t.v[1] - q * ptiles) * BP, q0 = q * BQ;
    return {x + ((int64_t)t.v[2] * d_in + p0) * kItem, grad_out + ((int64_t)t.v[2] * d_out + q0) * kItem, min(BP, d_in - p0),
            min(BQ, d_out - q0), t.v[3], e, p0, q0, t.v[1], t.v[4]};
  }
  __device__ __forceinline__ bool sums(const Place& at) const { return grad_bias != nullptr && at.p0 == 0; }
  __device__ __forceinline__ bool twice() const { return false; }
  __device__ __forceinline__ float4* partial_at(int slot, int tile, int i, int thread) const {
    return partial + (((int64_t)slot * ptiles * qtiles + tile) * (TILE::TP * TILE::TQ * 4) + i) * TILE::kThreads + thread;
  }
  __device__ __forceinline__ float* sums_at(int slot, int tile, int u, int thread) const {
    return partial_sums + (((int64_t)slot * ptiles * qtiles + tile) * TILE::TQ + u) * TILE::kThreads + thread;
  }

  __device__ __forceinline__ void finish(const Place& at, const TILE& tile) const {
    if (at.slot < 0) {
      store(at, tile);
      return;
    }
#pragma unroll
    for (int t = 0; t < TILE::TP; ++t)
#pragma unroll
      for (int u = 0; u < TILE::TQ; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          *partial_at(at.slot, at.tile, (t * TILE::TQ + u) * 4 + j, (int)threadIdx.x) =
              make_float4(tile.acc[t][u][4 * j], tile.acc[t][u][4 * j + 1], tile.acc[t][u][4 * j + 2], tile.acc[t][u][4 * j + 3]);
    if (sums(at))
#pragma unroll
      for (int u = 0; u < TILE::TQ; ++u) *sums_at(at.slot, at.tile, u, (int)threadIdx.x) = tile.sums[u];
  }

  __device__ __forceinline__ typename TILE::Lines lines(const Place& at, int wave) const {
    return TILE::lines(grad_w + (((int64_t)at.expert * d_out + at.q0) * d_in + at.p0) * kItem, (uint32_t)d_in * kItem, at.nq, at.np,
                       wave);
  }
  // The sums over Q of tile u of a wave: the waves of one column of waves have the same, the first stores them, the lane
  // halves' joined.
  __device__ __forceinline__ void store_sums(const Place& at, int wave, int u, float half) const {
    constexpr int kWP = BP / 32 / TILE::TP;
    const int lane = (int)threadIdx.x % 64, q = (wave / kWP * TILE::TQ + u) * 32 + lane;
    const float sum = half + __shfl_xor(half, 32, 64);
    if (wave % kWP != 0 || lane >= 32 || q >= at.nq) return;
    const int64_t i = (int64_t)at.expert * d_out + at.q0 + q;
    if (kItem == 4) reinterpret_cast<float*>(grad_bias)[i] = sum;
    else reinterpret_cast<__bf16*>(grad_bias)[i] = (__bf16)sum;
  }

  __device__ __forceinline__ void store(const Place& at, const TILE& tile) const {
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
    const typename TILE::Lines o = lines(at, wave);
#pragma unroll
    for (int g = 0; g < TILE::kGroups; ++g)
#pragma unroll
      for (int u = 0; u < TILE::TQ; ++u) {
        float v[16 * TILE::kGroupTiles];
        tile.results(g, u, v);
        // past the caches: 4096 rows of 64 experts, 1024 x 4096 weights each, 134 -> 100 us, 65536 rows 514 -> 508
        TILE::template put<true>(o, g, u, TILE::pack(v));
      }
    if (!sums(at)) return;
#pragma unroll
    for (int u = 0; u < TILE::TQ; ++u) store_sums(at, wave, u, tile.sums[u]);
  }

  // Adds up and stores group g, tile u of what wave `wave` of a tile's workgroup had of each part.
  __device__ __forceinline__ void join(const Place& at, const RowRange& range, int count, int wave, int g, int u) const {
    constexpr int kElems = 16 * TILE::kGroupTiles;
    const int thread = wave * 64 + (int)threadIdx.x % 64;
    const bool with_sums = sums(at) && g == 0;
    float v[kElems] = {}, sum = 0.0f;
#pragma unroll 2
    for (int k = 0; k < count; ++k) {
      const int slot = slot_of(part_start(range, count, k));
#pragma unroll
      for (int i = 0; i < kElems / 4; ++i) {
        const int t = g * TILE::kGroupTiles + i / 4;
        const float4 x = *partial_at(slot, at.tile, (t * TILE::TQ + u) * 4 + i % 4, thread);
        v[4 * i] += x.x;
        v[4 * i + 1] += x.y;
        v[4 * i + 2] += x.z;
        v[4 * i + 3] += x.w;
      }
      if (with_sums) sum += *sums_at(slot, at.tile, u, thread);
    }
    typename TILE::Lines o = lines(at, wave);
    // u and g are no constants here: the first group and tile of lines moved on to them
    o.at += (uint32_t)u * 32 * o.ld + 128u * g;
    o.p += 32 * TILE::kGroupTiles * g;
    TILE::put(o, 0, 0, TILE::pack(v));
    if (with_sums) store_sums(at, wave, u, sum);
  }
};

template <typename DT, typename TILE, int BP, int BQ, int PARTS>
__global__ __launch_bounds__(TILE::kThreads, 2) void weight_grad_kernel(const char* __restrict__ grad_out,
                                                                        const char* __restrict__ x,
                                                                        const int32_t* __restrict__ offsets, int rows, int d_in,
                                                                        int d_out, int E, char* __restrict__ grad_w,
                                                                        char* __restrict__ grad_bias, float4* partial,
                                                                        float* partial_sums, int slots) {
  const int ptiles = (d_in + BP - 1) / BP, qtiles = (d_out + BQ - 1) / BQ;
  // (without slots no expert is cut, whatever the offsets are)
  const RowParts parts(offsets, E, rows, slots == 0 ? max(rows, kLeastPart) : part_rows(rows_of(offsets, E - 1, rows).hi, ptiles * qtiles, PARTS));
  const WeightGradJob<DT, TILE, BP, BQ> job = {grad_out, x, grad_w, grad_bias, partial, partial_sums, d_in, d_out, ptiles, qtiles,
                                               slots, parts};
  // an XCD's tiles are consecutive ones with an eighth of the work
  const RowRange mine = parts.run_of_work((int)(blockIdx.x % 8), 8, ptiles * qtiles);
  TILE tile;
  tile.run(job, mine.lo + (int)(blockIdx.x / 8), mine.hi, (int)(gridDim.x / 8));
}

// Adds up the parts of the experts that were cut: a wave takes a group's results of one wave of a tile's workgroup.  It looks at 64
// of them at a time; most calls have none that were cut.
constexpr int kJoinThreads = 256;
template <typename DT, typename TILE, int BP, int BQ, int PARTS>
__global__ __launch_bounds__(kJoinThreads) void join_parts_kernel(const int32_t* __restrict__ offsets, int rows, int d_in,
                                                                  int d_out, int E, char* __restrict__ grad_w,
                                                                  char* __restrict__ grad_bias, float4* partial,
                                                                  float* partial_sums, int slots) {
  const int ptiles = (d_in + BP - 1) / BP, qtiles = (d_out + BQ - 1) / BQ, tiles = ptiles * qtiles;
  const RowParts parts(offsets, E, rows, part_rows(rows_of(offsets, E - 1, rows).hi, tiles, PARTS));
  if (parts.total == E) return;            // no expert was cut
  const WeightGradJob<DT, TILE, BP, BQ> job = {nullptr, nullptr, grad_w, grad_bias, partial, partial_sums, d_in, d_out, ptiles,
                                               qtiles, slots, parts};
  constexpr int kShares = TILE::kWaves * TILE::kGroups * TILE::TQ;     // of a tile
  // Number i is share i % kShares of tile i / kShares; a wave's lanes look at the tiles of 64 numbers, its own ones.
  const int lane = (int)threadIdx.x % kWave;
  const int64_t waves = (int64_t)gridDim.x * (kJoinThreads / kWave), all = (int64_t)parts.total * tiles * kShares;
  const int64_t self = (int64_t)blockIdx.x * (kJoinThreads / kWave) + __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
  for (int64_t i0 = self; i0 < all; i0 += waves * kWave) {
    const int64_t i = min(i0 + lane * waves, all - 1);
    const int n = (int)(i / kShares);
    const int m = (int)((uint32_t)n / (uint32_t)tiles);
    const RowParts::Found f = parts.find(m);
    const TileEntry entry = job.entry_of(f, n - m * tiles);
    uint64_t cut = __ballot(f.count > 1 && f.number == 0 && i0 + lane * waves < all);
    while (cut != 0) {
      const int at = __builtin_ctzll(cut);
      cut &= cut - 1;
      TileEntry e;
#pragma unroll
      for (int j = 0; j < 5; ++j) e.v[j] = __builtin_amdgcn_readlane(entry.v[j], at);
      const RowRange range = {__builtin_amdgcn_readlane(f.range.lo, at), __builtin_amdgcn_readlane(f.range.hi, at)};
      const int share = (int)((i0 + at * waves) % kShares);
      job.join(job.place(e), range, __builtin_amdgcn_readlane(f.count, at), share % TILE::kWaves, share / TILE::kWaves % TILE::kGroups,
               share / TILE::kWaves / TILE::kGroups);
    }
  }
}

template <typename DT, typename S>
hipError_t forward_on_tiles(const void* x, const void* w, const void* bias, const int32_t* offsets, int64_t rows, int d_in,
                            int d_out, int E, int act, void* pre, void* out, hipStream_t stream) {
  typedef Tile<DT, DT, false, false, S::BP, S::BQ, S::WP, S::WQ> TILE;
  auto kernel = forward_kernel<DT, DT, TILE, S::BP, S::BQ>;
  if (hipError_t e = allow_lds(kernel, TILE::kLds); e != hipSuccess) return e;
  const uint64_t tiles = (uint64_t)most_row_tiles(rows, E, S::BQ) * ((d_out + S::BP - 1) / S::BP);
  kernel<<<blocks_for(tiles, S::kPerUnit), TILE::kThreads, TILE::kLds, stream>>>(
      (const char*)x, (const char*)w, nullptr, nullptr, (const char*)bias, offsets, (int)rows, d_in, d_out, E, act, (char*)pre,
      (char*)out);
  return hipGetLastError();
}

// binary32's tiles take 16 times as long: few rows are up to 32 (512 rows, 768 -> 2048 columns of 16 experts 38.6 and 57 us, 1024
// rows 61.5 and 56).
template <typename DT>
hipError_t forward(const void* x, const void* w, const void* bias, const int32_t* offsets, int64_t rows, int d_in, int d_out,
                   int E, int act, void* pre, void* out, hipStream_t stream) {
  constexpr bool kWide = std::is_same<DT, F32>::value;
  if (few_rows(rows, E, d_out, kWide ? 32 : 8))
    return launch_direct<DT, DT>((const char*)x, (const char*)w, nullptr, nullptr, (const char*)bias, offsets, rows,
                                 d_in * ItemSize<DT>::value, d_out, E, act, (char*)pre, (char*)out, stream);
  if constexpr (!kWide)
    if (!small_tiles(rows, E, d_out))
      return forward_on_tiles<DT, Large>(x, w, bias, offsets, rows, d_in, d_out, E, act, pre, out, stream);
  return forward_on_tiles<DT, Small>(x, w, bias, offsets, rows, d_in, d_out, E, act, pre, out, stream);
}

template <typename DT, typename S>
hipError_t input_grad_on_tiles(const void* grad_out, const void* w, const int32_t* offsets, int64_t rows, int d_in, int d_out,
                               int E, int act, const void* pre, void* grad_x, hipStream_t stream) {
  typedef Tile<DT, DT, true, false, S::BP, S::BQ, S::WP, S::WQ> TILE;
  auto kernel = input_grad_kernel<DT, TILE, S::BP, S::BQ>;
  if (hipError_t e = allow_lds(kernel, TILE::kLds); e != hipSuccess) return e;
  const uint64_t tiles = (uint64_t)most_row_tiles(rows, E, S::BQ) * ((d_in + S::BP - 1) / S::BP);
  kernel<<<blocks_for(tiles, S::kPerUnit), TILE::kThreads, TILE::kLds, stream>>>(
      (const char*)grad_out, (const char*)w, offsets, (int)rows, d_in, d_out, E, act, (const char*)pre, (char*)grad_x);
  return hipGetLastError();
}

template <typename DT>
hipError_t input_grad(const void* grad_out, const void* w, const int32_t* offsets, int64_t rows, int d_in, int d_out, int E,
                      int act, const void* pre, void* grad_x, hipStream_t stream) {
  if constexpr (!std::is_same<DT, F32>::value)
    if (!small_tiles(rows, E, d_in))
      return input_grad_on_tiles<DT, Large>(grad_out, w, offsets, rows, d_in, d_out, E, act, pre, grad_x, stream);
  return input_grad_on_tiles<DT, Small>(grad_out, w, offsets, rows, d_in, d_out, E, act, pre, grad_x, stream);
}

template <typename DT> struct WeightGradPlan {
  typedef WeightGradShape<DT> S;
  typedef Tile<DT, DT, true, true, S::BP, S::BQ, S::WP, S::WQ> TILE;
  uint64_t tiles;         // of an expert
  bool cut;               // there may be experts in parts
  uint64_t slots;         // of partial sums
  size_t off_sums, total_bytes;

  WeightGradPlan(int64_t rows, int d_in, int d_out) {
    tiles = (uint64_t)((d_in + S::BP - 1) / S::BP) * ((d_out + S::BQ - 1) / S::BQ);
    cut = rows > kLeastPart && tiles < S::PARTS;          // with as many tiles a part is all rows
    slots = cut ? part_slots(rows, tiles, S::PARTS) : 0;
    off_sums = slots * tiles * S::BP * S::BQ * 4;
    total_bytes = off_sums + slots * tiles * TILE::TQ * TILE::kThreads * 4;
  }
};

template <typename DT>
hipError_t weight_grad(const void* grad_out, const void* x, const int32_t* offsets, int64_t rows, int d_in, int d_out, int E,
                       void* grad_w, void* grad_bias, char* workspace, hipStream_t stream) {
  typedef WeightGradShape<DT> S;
  typedef typename WeightGradPlan<DT>::TILE TILE;
  const WeightGradPlan<DT> plan(rows, d_in, d_out);
  auto kernel = weight_grad_kernel<DT, TILE, S::BP, S::BQ, S::PARTS>;
  if (hipError_t e = allow_lds(kernel, TILE::kLds); e != hipSuccess) return e;
  float4* const partial = (float4*)workspace;
  float* const sums = (float*)(workspace + plan.off_sums);
  const uint64_t parts = (uint64_t)E + (plan.cut ? rows / (kLeastPart / 2) : 0);
  kernel<<<blocks_for(parts * plan.tiles, S::kPerUnit), TILE::kThreads, TILE::kLds, stream>>>(
      (const char*)grad_out, (const char*)x, offsets, (int)rows, d_in, d_out, E, (char*)grad_w, (char*)grad_bias, partial, sums, (int)plan.slots);
  if (hipError_t e = hipGetLastError(); e != hipSuccess || !plan.cut) return e;
  join_parts_kernel<DT, TILE, S::BP, S::BQ, S::PARTS><<<2 * kUnits, kJoinThreads, 0, stream>>>(
      offsets, (int)rows, d_in, d_out, E, (char*)grad_w, (char*)grad_bias, partial, sums, (int)plan.slots);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_expert_forward(const void* x, const void* w, const void* bias, const int32_t* offsets, int64_t rows,
                                 int d_in, int d_out, int E, bool bf16, int act, void* pre, void* out, hipStream_t stream) {
  return bf16 ? forward<BF16>(x, w, bias, offsets, rows, d_in, d_out, E, act, pre, out, stream)
              : forward<F32>(x, w, bias, offsets, rows, d_in, d_out, E, act, pre, out, stream);
}

hipError_t launch_expert_input_grad(const void* grad_out, const void* w, const int32_t* offsets, int64_t rows, int d_in,
                                    int d_out, int E, bool bf16, int act, const void* pre, void* grad_x, hipStream_t stream) {
  return bf16 ? input_grad<BF16>(grad_out, w, offsets, rows, d_in, d_out, E, act, pre, grad_x, stream)
              : input_grad<F32>(grad_out, w, offsets, rows, d_in, d_out, E, act, pre, grad_x, stream);
}

size_t expert_workspace_bytes(int64_t rows, int d_in, int d_out, bool bf16) {
  return bf16 ? WeightGradPlan<BF16>(rows, d_in, d_out).total_bytes : WeightGradPlan<F32>(rows, d_in, d_out).total_bytes;
}

hipError_t launch_expert_weight_grad(const void* grad_out, const void* x, const int32_t* offsets, int64_t rows, int d_in,
                                     int d_out, int E, bool bf16, void* grad_w, void* grad_bias, char* workspace,
                                     hipStream_t stream) {
  return bf16 ? weight_grad<BF16>(grad_out, x, offsets, rows, d_in, d_out, E, grad_w, grad_bias, workspace, stream)
              : weight_grad<F32>(grad_out, x, offsets, rows, d_in, d_out, E, grad_w, grad_bias, workspace, stream);
}

}  // namespace lshmoe
