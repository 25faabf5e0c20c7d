// Products of few rows per expert: out[q][p] = act(sum_k x[q][k] W_e[p][k] + b_e[p]) with the operands straight from memory into
// registers.
//
// With few rows the weights are read once and are all that counts, so the waves are made many and small: a wave has 16 columns
// and 16 TQ rows, KS waves share them by k and join their sums in LDS, in the order of k.  Loads of the next steps are under
// way while a step's products run.  A workgroup takes up to 4 of its columns' turns after one look at the offsets.  Bound by
// the read of the weights: 74 rows of 16 experts, 768 -> 2048 columns of bf16 take 13.1 us, 3.8 TB/s; 4 bits 8.2 us.
#pragma once

#include "kernels.h"
#include "rows_by_expert.h"

namespace lshmoe {

namespace {

typedef float direct_f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 direct_bf16x8 __attribute__((ext_vector_type(8)));
typedef int direct_i32x8 __attribute__((ext_vector_type(8)));

// c += W x^T of one step, 64 bytes of a row: lane l has the piece l / 16 of row l % 16.
template <typename OT> __device__ __forceinline__ void direct_mma(const u32x4& a, const u32x4& b, uint32_t scale_a,
                                                                  uint32_t scale_b, direct_f32x4& c) {
  if constexpr (std::is_same<OT, BF16>::value) {
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(direct_bf16x8, a), __builtin_bit_cast(direct_bf16x8, b), c, 0, 0, 0);
  } else if constexpr (std::is_same<OT, F32>::value) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[i]), __uint_as_float(b[i]), c, 0, 0, 0);
  } else {
    const direct_i32x8 wide_a = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
    const direct_i32x8 wide_b = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
    c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide_a, wide_b, c, 4, 4, 0, (int)scale_a, 0, (int)scale_b);
  }
}

// 16 bytes, or zeros behind the end of the buffer.
__device__ __forceinline__ u32x4 direct_load16(const __amdgpu_buffer_rsrc_t& buffer, uint32_t at) {
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(buffer, (int)at, 0, 0));
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t direct_buffer(const char* base, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, (int)min(bytes, (int64_t)0x7fffffff), 0x00020000);
}

template <typename OT, typename DT, int TQ, int KS>
__global__ __launch_bounds__(256) void direct_kernel(const char* __restrict__ x, const char* __restrict__ w,
                                                     const char* __restrict__ x_scales, const char* __restrict__ w_scales,
                                                     const char* __restrict__ bias, const int32_t* __restrict__ offsets, int rows,
                                                     int line, int d_out, int E, int act, int turns, char* __restrict__ pre,
                                                     char* __restrict__ out) {
  constexpr bool kScaled = std::is_same<OT, MX4>::value;
  constexpr int kColumns = 16 * 4 / KS, kAhead = 4, kItem = ItemSize<DT>::value;
  constexpr uint32_t kBehind = 0x80000000u;                  // an offset behind the end of every buffer
  __shared__ direct_f32x4 parts[KS > 1 ? 4 : 1][TQ][64];
  const RowTiles tiles(offsets, E, rows, 16 * TQ);
  const int ptiles = (d_out + turns * kColumns - 1) / (turns * kColumns);
  if (linear_block() >= (uint64_t)tiles.total * ptiles) return;
  const RowTile t = tiles.tile((int)linear_block(), ptiles);
  const int expert = __builtin_amdgcn_readfirstlane(t.expert), first = __builtin_amdgcn_readfirstlane(t.first);
  const int nq = __builtin_amdgcn_readfirstlane(t.rows);
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64), part = wave % KS;
  const int lane = (int)threadIdx.x % 64, r = lane % 16, g = lane / 16;

  for (int turn = 0; turn < turns; ++turn) {
    const int p0 = (__builtin_amdgcn_readfirstlane(t.column) * turns + turn) * kColumns + wave / KS * 16, np = min(16, d_out - p0);
    // Pieces of 16 bytes: W's row p0 + r, x's rows 16 u + r.  A row ends at `line` bytes, the buffers where their last row does.
    const int64_t column = (int64_t)expert * d_out + p0;
    const __amdgpu_buffer_rsrc_t wb = direct_buffer(w + column * line, np <= 0 ? 0 : (int64_t)np * line);
    const __amdgpu_buffer_rsrc_t xb = direct_buffer(x + (int64_t)first * line, (int64_t)nq * line);
    const int blocks = line / 16;                              // scaled: blocks of a row, a scale byte each
    const char* const ws = kScaled ? w_scales + (column + min(r, max(np, 1) - 1)) * blocks : nullptr;
    const int steps = (line + 63) / 64, from = steps * part / KS, to = steps * (part + 1) / KS;

    u32x4 a[2][kAhead], b[2][kAhead][TQ];
    uint32_t sa[2][kAhead], sb[2][kAhead][TQ];
    auto load = [&](int buf, int s0) {
  #pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int s = s0 + i;
        const uint32_t piece = (uint32_t)(64 * s + 16 * g);
        const bool there = s < to && (int)piece < line;
        a[buf][i] = direct_load16(wb, there ? r * (uint32_t)line + piece : kBehind);
  #pragma unroll
        for (int u = 0; u < TQ; ++u) b[buf][i][u] = direct_load16(xb, there ? (16 * u + r) * (uint32_t)line + piece : kBehind);
        if (kScaled) {
          const int block = there && np > 0 ? 4 * s + g : 0;   // where there is no piece, any of the row's scales that is no NaN
          sa[buf][i] = there && np > 0 ? (uint32_t)(uint8_t)ws[block] : 127u;
  #pragma unroll
          for (int u = 0; u < TQ; ++u)
            sb[buf][i][u] = there && 16 * u + r < nq ? (uint32_t)(uint8_t)x_scales[((int64_t)first + 16 * u + r) * blocks + block] : 127u;
        }
      }
    };
    direct_f32x4 acc[TQ] = {};
    auto multiply = [&](int buf) {
  #pragma unroll
      for (int i = 0; i < kAhead; ++i)
  #pragma unroll
        for (int u = 0; u < TQ; ++u) direct_mma<OT>(a[buf][i], b[buf][i][u], sa[buf][i], sb[buf][i][u], acc[u]);
    };
    load(0, from);
    for (int s = from; s < to; s += 2 * kAhead) {
      load(1, s + kAhead);
      multiply(0);
      load(0, s + 2 * kAhead);
      multiply(1);
    }

    if (KS > 1) {
      if (part > 0)
  #pragma unroll
        for (int u = 0; u < TQ; ++u) parts[wave][u][lane] = acc[u];
      __syncthreads();
  #pragma unroll
      for (int i = 1; i < KS; ++i)
  #pragma unroll
        for (int u = 0; u < TQ; ++u) acc[u] += parts[(wave + i) % 4][u][lane];
      __syncthreads();
      if (part > 0) continue;
    }
    // a lane has 4 consecutive columns of one row; d_out is a multiple of 4
    const int p = p0 + 4 * g;
    if (p >= d_out) continue;
    auto store4 = [&](char* at, const float (&v)[4]) {
      if (kItem == 2) *reinterpret_cast<uint2*>(at) = make_uint2(f32_to_bf16_pair(v[0], v[1]), f32_to_bf16_pair(v[2], v[3]));
      else *reinterpret_cast<float4*>(at) = make_float4(v[0], v[1], v[2], v[3]);
    };
    float add[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (bias) {
      const char* at = bias + ((int64_t)expert * d_out + p) * kItem;
  #pragma unroll
      for (int j = 0; j < 4; ++j)
        add[j] = kItem == 2 ? (float)reinterpret_cast<const __bf16*>(at)[j] : reinterpret_cast<const float*>(at)[j];
    }
  #pragma unroll
    for (int u = 0; u < TQ; ++u) {
      const int q = 16 * u + r;
      if (q >= nq) continue;
      const int64_t at = (((int64_t)first + q) * d_out + p) * kItem;
      float v[4];
  #pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = acc[u][j] + add[j];
      if (pre) store4(pre + at, v);
  #pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = activate<DT>(v[j], act);
      store4(out + at, v);
    }
  }
}

// line: bytes of a row of x and W.
template <typename OT, typename DT>
hipError_t launch_direct(const char* x, const char* w, const char* x_scales, const char* w_scales, const char* bias,
                         const int32_t* offsets, int64_t rows, int line, int d_out, int E, int act, char* pre, char* out,
                         hipStream_t stream) {
  auto run = [&](auto tq, auto ks) {
    constexpr int TQ = decltype(tq)::value, KS = decltype(ks)::value;
    const uint64_t row_tiles = most_row_tiles(rows, E, 16 * TQ), columns = (d_out + 16 * 4 / KS - 1) / (16 * 4 / KS);
    int turns = 1;
    while (turns < 4 && row_tiles * columns > 2048ull * turns) turns *= 2;
    direct_kernel<OT, DT, TQ, KS><<<grid_of_blocks(row_tiles * ((columns + turns - 1) / turns)), 256, 0, stream>>>(
        x, w, x_scales, w_scales, bias, offsets, (int)rows, line, d_out, E, act, turns, pre, out);
    return hipGetLastError();
  };
  // Waves enough to have the card's memory busy: k is split while there are fewer than 16 to a compute unit and 16 steps to a part.
  auto split = [&](auto tq) {
    constexpr int TQ = decltype(tq)::value;
    const uint64_t waves = (uint64_t)most_row_tiles(rows, E, 16 * TQ) * ((d_out + 15) / 16);
    if (waves * 2 <= 4096 && line >= 4 * 16 * 64) return run(tq, std::integral_constant<int, 4>{});
    if (waves <= 4096 && line >= 2 * 16 * 64) return run(tq, std::integral_constant<int, 2>{});
    return run(tq, std::integral_constant<int, 1>{});
  };
  if (rows <= 16 * (int64_t)E) return split(std::integral_constant<int, 1>{});
  if (rows <= 32 * (int64_t)E) return split(std::integral_constant<int, 2>{});
  return split(std::integral_constant<int, 4>{});
}

}  // namespace

}  // namespace lshmoe
