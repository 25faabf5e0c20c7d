// The experts' products on rows that are grouped by expert: rows expert_offsets[e] .. expert_offsets[e+1] - 1 belong to
// expert e.  The offsets are in device memory, so a launch is sized for the worst case and a workgroup finds its expert
// and its rows from the offsets itself.
//
//   forward      pre = x W_e^T + b_e,  out = act(pre)          W_e [d_out, d_in]
//   input        grad_x = (grad_out W_e) * act'(pre)
//   weight       grad_W_e = grad_out_e^T x_e,  grad_b_e = sum of grad_out_e
//
// The tiles and how they are computed: product_tile.h.
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
  __device__ __forceinline__ TileEntry entry(int n) const {
    const RowTile t = tiles.find(n, ptiles);
    return {{t.expert, t.first, t.rows, t.column * BP}};
  }
  __device__ __forceinline__ Place place(const TileEntry& t) const {
    const int expert = t.v[0], first = t.v[1], nq = t.v[2], p0 = t.v[3];
    return {w + ((int64_t)expert * d_out * d_in + p0) * kItem, grad_out + (int64_t)first * d_out * kItem, nullptr, nullptr,
            min(BP, d_in - p0), nq, d_out, TILE::OpP::kChunk, expert, first, p0};
  }
  __device__ __forceinline__ bool sums(const Place&) const { return false; }
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
            for (int i = 0; i < kElems; ++i) v[i] *= activation_slope(z[i], ACT);
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

template <typename DT, typename TILE, int BP, int BQ> struct WeightGradJob {
  struct Place {
    const char *p, *q;
    int np, nq, K, expert, p0, q0;
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
  const int32_t* offsets;
  int rows, d_in, d_out, E, ptiles, qtiles;

  __device__ __forceinline__ uint32_t p_stride() const { return (uint32_t)d_in * kItem; }
  __device__ __forceinline__ uint32_t q_stride() const { return (uint32_t)d_out * kItem; }
  __device__ __forceinline__ uint32_t s_stride() const { return 0; }
  __device__ __forceinline__ TileEntry entry(int n) const {
    const int e = min((int)((uint32_t)n / (uint32_t)(ptiles * qtiles)), E - 1);
    const RowRange range = rows_of(offsets, e, rows);
    return {{e, n - e * ptiles * qtiles, range.lo, range.hi - range.lo}};
  }
  __device__ __forceinline__ Place place(const TileEntry& t) const {
    const int e = t.v[0], q = (int)((uint32_t)t.v[1] / (uint32_t)ptiles), p0 = (t.v[1] - q * ptiles) * BP, q0 = q * BQ;
    return {x + ((int64_t)t.v[2] * d_in + p0) * kItem, grad_out + ((int64_t)t.v[2] * d_out + q0) * kItem, min(BP, d_in - p0),
            min(BQ, d_out - q0), t.v[3], e, p0, q0};
  }
  __device__ __forceinline__ bool sums(const Place& at) const { return grad_bias != nullptr && at.p0 == 0; }
  __device__ __forceinline__ void finish(const Place& at, const TILE& tile) const {
    const typename TILE::Lines o = TILE::lines(grad_w + (((int64_t)at.expert * d_out + at.q0) * d_in + at.p0) * kItem,
                                               (uint32_t)d_in * kItem, at.nq, at.np);
#pragma unroll
    for (int g = 0; g < TILE::kGroups; ++g)
#pragma unroll
      for (int u = 0; u < TILE::TQ; ++u) {
        float v[16 * TILE::kGroupTiles];
        tile.results(g, u, v);
        TILE::put(o, g, u, TILE::pack(v));
      }
    if (!sums(at)) return;
    // the waves of one column of waves have the same Q: the first stores, the lane halves' sums joined
    constexpr int kWP = BP / 32 / TILE::TP;
    const int lane = (int)threadIdx.x % 64, wave = (int)threadIdx.x / 64;
#pragma unroll
    for (int u = 0; u < TILE::TQ; ++u) {
      const float sum = tile.sums[u] + __shfl_xor(tile.sums[u], 32, 64);
      const int q = (wave / kWP * TILE::TQ + u) * 32 + lane;
      if (wave % kWP != 0 || lane >= 32 || q >= at.nq) continue;
      const int64_t i = (int64_t)at.expert * d_out + at.q0 + q;
      if (kItem == 4) reinterpret_cast<float*>(grad_bias)[i] = sum;
      else reinterpret_cast<__bf16*>(grad_bias)[i] = (__bf16)sum;
    }
  }
};

template <typename DT, typename TILE, int BP, int BQ>
__global__ __launch_bounds__(TILE::kThreads, 2) void weight_grad_kernel(const char* __restrict__ grad_out,
                                                                        const char* __restrict__ x,
                                                                        const int32_t* __restrict__ offsets, int rows, int d_in,
                                                                        int d_out, int E, char* __restrict__ grad_w,
                                                                        char* __restrict__ grad_bias) {
  const int ptiles = (d_in + BP - 1) / BP, qtiles = (d_out + BQ - 1) / BQ;
  const WeightGradJob<DT, TILE, BP, BQ> job = {grad_out, x, grad_w, grad_bias, offsets, rows, d_in, d_out, E, ptiles, qtiles};
  const Share s = share_of_block(E * ptiles * qtiles);
  TILE tile;
  tile.run(job, s.first, s.end, s.step);
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

// Rows per expert that a call can have at most on average decide.  Up to 8 (binary32: 32): waves that read the weights for
// themselves (768 -> 2048 columns of 16 experts: 74 rows 13.1 and 13.9 us on tiles, 2048 -> 768 13.1 and 22.9; 256 rows 15.6
// and 13.8; binary32, 512 rows 38.6 and 57, 1024 rows 61.5 and 56).  Up to 128: small tiles (1024 -> 4096 columns of 16
// experts, 2048 rows 28.7 us and 34 on large ones, 4096 rows 43.3 and 39.5).
template <typename DT>
hipError_t forward(const void* x, const void* w, const void* bias, const int32_t* offsets, int64_t rows, int d_in, int d_out,
                   int E, int act, void* pre, void* out, hipStream_t stream) {
  constexpr bool kWide = std::is_same<DT, F32>::value;
  if (rows <= (kWide ? 32 : 8) * (int64_t)E)
    return launch_direct<DT, DT>((const char*)x, (const char*)w, nullptr, nullptr, (const char*)bias, offsets, rows,
                                 d_in * ItemSize<DT>::value, d_out, E, act, (char*)pre, (char*)out, stream);
  if constexpr (!kWide)
    if (rows > 128 * (int64_t)E)
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
    if (rows > 128 * (int64_t)E)
      return input_grad_on_tiles<DT, Large>(grad_out, w, offsets, rows, d_in, d_out, E, act, pre, grad_x, stream);
  return input_grad_on_tiles<DT, Small>(grad_out, w, offsets, rows, d_in, d_out, E, act, pre, grad_x, stream);
}

template <typename DT>
hipError_t weight_grad(const void* grad_out, const void* x, const int32_t* offsets, int64_t rows, int d_in, int d_out, int E,
                       void* grad_w, void* grad_bias, hipStream_t stream) {
  typedef typename std::conditional<std::is_same<DT, F32>::value, Small, Large>::type S;
  typedef Tile<DT, DT, true, true, S::BP, S::BQ, S::WP, S::WQ> TILE;
  auto kernel = weight_grad_kernel<DT, TILE, S::BP, S::BQ>;
  if (hipError_t e = allow_lds(kernel, TILE::kLds); e != hipSuccess) return e;
  const uint64_t tiles = (uint64_t)E * ((d_in + S::BP - 1) / S::BP) * ((d_out + S::BQ - 1) / S::BQ);
  kernel<<<blocks_for(tiles, S::kPerUnit), TILE::kThreads, TILE::kLds, stream>>>(
      (const char*)grad_out, (const char*)x, offsets, (int)rows, d_in, d_out, E, (char*)grad_w, (char*)grad_bias);
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

size_t expert_workspace_bytes(int64_t, int, int, int, bool) { return 0; }

hipError_t launch_expert_weight_grad(const void* grad_out, const void* x, const int32_t* offsets, int64_t rows, int d_in,
                                     int d_out, int E, bool bf16, void* grad_w, void* grad_bias, char*, hipStream_t stream) {
  return bf16 ? weight_grad<BF16>(grad_out, x, offsets, rows, d_in, d_out, E, grad_w, grad_bias, stream)
              : weight_grad<F32>(grad_out, x, offsets, rows, d_in, d_out, E, grad_w, grad_bias, stream);
}

}  // namespace lshmoe
