// The experts' products on rows that are grouped by expert: rows expert_offsets[e] .. expert_offsets[e+1] - 1 belong to
// expert e.  The offsets are in device memory, so a launch is sized for the worst case and a workgroup finds its expert
// and its rows from the offsets itself.
//
//   forward      pre = x W_e^T + b_e,  out = act(pre)          W_e [d_out, d_in]
//   input        grad_x = (grad_out W_e) * act'(pre)
//   weight       grad_W_e = grad_out_e^T x_e,  grad_b_e = sum of grad_out_e
//
// All three are out[q][p] = sum_k Q[q][k] P[p][k], p the index that is contiguous in the output:
//   forward      q = row, p = d_out, k = d_in       Q = x, P = W_e, both contiguous in k
//   input        q = row, p = d_in,  k = d_out      Q = grad_out contiguous in k, P = W_e contiguous in p
//   weight       q = d_out, p = d_in, k = row       Q = grad_out contiguous in q, P = x contiguous in p
// The matrix instruction takes P as its first operand: a lane then holds consecutive p of one q.
#include "kernels.h"
#include "rows_by_expert.h"

namespace lshmoe {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kTile = 64, kChunk = 32;   // outputs of a workgroup in either direction, k per step

template <typename DT> struct Elem;
template <> struct Elem<F32> {
  typedef float type;
  static __device__ __forceinline__ float widen(float v) { return v; }
  static __device__ __forceinline__ float narrow(float v) { return v; }
};
template <> struct Elem<BF16> {
  typedef __bf16 type;
  static __device__ __forceinline__ float widen(__bf16 v) { return (float)v; }
  static __device__ __forceinline__ __bf16 narrow(float v) { return (__bf16)v; }
};

template <typename DT> __device__ __forceinline__ void mma(const uint4& a, const uint4& b, f32x4& c);
template <> __device__ __forceinline__ void mma<BF16>(const uint4& a, const uint4& b, f32x4& c) {
  c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ void mma<F32>(const uint4& a, const uint4& b, f32x4& c) {
  c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.x), __uint_as_float(b.x), c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.y), __uint_as_float(b.y), c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.z), __uint_as_float(b.z), c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.w), __uint_as_float(b.w), c, 0, 0, 0);
}

template <typename DT> struct Operand {
  const typename Elem<DT>::type* base;   // element (index 0, k 0) of the tile
  int64_t index_stride, k_stride;
  int indices;                           // of the tile that exist
};

// One tile of out = Q P^T; store(q, p, value) takes the results, sum(q, value) the sums of Q over k where wanted.
template <typename DT, typename Store, typename Sum>
__device__ __forceinline__ void tile_product(const Operand<DT>& P, const Operand<DT>& Q, int K, bool sums, Store&& store,
                                             Sum&& sum) {
  typedef typename Elem<DT>::type T;
  constexpr int kPiece = 16 / sizeof(T), kPad = kChunk + kPiece;
  __shared__ __align__(16) T lp[kTile][kPad];
  __shared__ __align__(16) T lq[kTile][kPad];
  const int tid = (int)threadIdx.x, lane = tid % 64, wave = tid / 64, r = lane % 16, g = lane / 16;
  f32x4 acc[4] = {};
  float total = 0.0f;
  for (int k0 = 0; k0 < K; k0 += kChunk) {
    __syncthreads();
    for (int i = tid; i < kTile * kChunk; i += 256) {
      const int kp = P.k_stride == 1 ? i % kChunk : i / kTile, ip = P.k_stride == 1 ? i / kChunk : i % kTile;
      lp[ip][kp] = ip < P.indices && k0 + kp < K ? P.base[ip * P.index_stride + (int64_t)(k0 + kp) * P.k_stride] : (T)0.0f;
      const int kq = Q.k_stride == 1 ? i % kChunk : i / kTile, iq = Q.k_stride == 1 ? i / kChunk : i % kTile;
      lq[iq][kq] = iq < Q.indices && k0 + kq < K ? Q.base[iq * Q.index_stride + (int64_t)(k0 + kq) * Q.k_stride] : (T)0.0f;
    }
    __syncthreads();
    for (int s = 0; s < kChunk / (4 * kPiece); ++s) {
      const uint4 b = *reinterpret_cast<const uint4*>(&lq[16 * wave + r][(4 * s + g) * kPiece]);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        mma<DT>(*reinterpret_cast<const uint4*>(&lp[16 * i + r][(4 * s + g) * kPiece]), b, acc[i]);
    }
    if (sums && tid < kTile)
      for (int k = 0; k < kChunk; ++k) total += Elem<DT>::widen(lq[tid][k]);
  }
  const int q = 16 * wave + r;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int p = 16 * i + 4 * g + j;
      if (q < Q.indices && p < P.indices) store(q, p, acc[i][j]);
    }
  if (sums && tid < kTile && tid < Q.indices) sum(tid, total);
}

template <typename DT>
__global__ __launch_bounds__(256) void forward_kernel(const void* x, const void* w, const void* bias,
                                                      const int32_t* __restrict__ offsets, int64_t rows, int d_in, int d_out,
                                                      int E, int act, void* pre, void* out) {
  typedef typename Elem<DT>::type T;
  const RowTile t = find_row_tile(offsets, E, rows, kTile, (int64_t)linear_block() / ((d_out + kTile - 1) / kTile));
  if (t.expert < 0) return;
  const int p0 = (int)(linear_block() % ((d_out + kTile - 1) / kTile)) * kTile;
  const Operand<DT> Q = {(const T*)x + t.first * d_in, d_in, 1, (int)min((int64_t)kTile, t.end - t.first)};
  const Operand<DT> P = {(const T*)w + ((int64_t)t.expert * d_out + p0) * d_in, d_in, 1, min(kTile, d_out - p0)};
  tile_product<DT>(P, Q, d_in, false, [&](int q, int p, float v) {
    if (bias) v += Elem<DT>::widen(((const T*)bias)[(int64_t)t.expert * d_out + p0 + p]);
    const int64_t at = (t.first + q) * d_out + p0 + p;
    if (pre) ((T*)pre)[at] = Elem<DT>::narrow(v);
    ((T*)out)[at] = Elem<DT>::narrow(activate(v, act));
  }, [](int, float) {});
}

template <typename DT>
__global__ __launch_bounds__(256) void input_grad_kernel(const void* grad_out, const void* w,
                                                         const int32_t* __restrict__ offsets, int64_t rows, int d_in,
                                                         int d_out, int E, int act, const void* pre, void* grad_x) {
  typedef typename Elem<DT>::type T;
  const RowTile t = find_row_tile(offsets, E, rows, kTile, (int64_t)linear_block() / ((d_in + kTile - 1) / kTile));
  if (t.expert < 0) return;
  const int p0 = (int)(linear_block() % ((d_in + kTile - 1) / kTile)) * kTile;
  const Operand<DT> Q = {(const T*)grad_out + t.first * d_out, d_out, 1, (int)min((int64_t)kTile, t.end - t.first)};
  const Operand<DT> P = {(const T*)w + (int64_t)t.expert * d_out * d_in + p0, 1, d_in, min(kTile, d_in - p0)};
  tile_product<DT>(P, Q, d_out, false, [&](int q, int p, float v) {
    const int64_t at = (t.first + q) * d_in + p0 + p;
    if (act != LSHMOE_ACT_NONE) v *= activation_slope(Elem<DT>::widen(((const T*)pre)[at]), act);
    ((T*)grad_x)[at] = Elem<DT>::narrow(v);
  }, [](int, float) {});
}

template <typename DT>
__global__ __launch_bounds__(256) void weight_grad_kernel(const void* grad_out, const void* x,
                                                          const int32_t* __restrict__ offsets, int64_t rows, int d_in,
                                                          int d_out, void* grad_w, void* grad_bias) {
  typedef typename Elem<DT>::type T;
  const int ptiles = (d_in + kTile - 1) / kTile, qtiles = (d_out + kTile - 1) / kTile;
  const uint64_t block = linear_block();
  const int64_t e = block / ((uint64_t)ptiles * qtiles);
  const int p0 = (int)(block % ptiles) * kTile, q0 = (int)(block / ptiles % qtiles) * kTile;
  const RowRange range = rows_of(offsets, (int)e, rows);
  const Operand<DT> Q = {(const T*)grad_out + range.lo * d_out + q0, 1, d_out, min(kTile, d_out - q0)};
  const Operand<DT> P = {(const T*)x + range.lo * d_in + p0, 1, d_in, min(kTile, d_in - p0)};
  tile_product<DT>(P, Q, (int)(range.hi - range.lo), grad_bias != nullptr && p0 == 0, [&](int q, int p, float v) {
    ((T*)grad_w)[((int64_t)e * d_out + q0 + q) * d_in + p0 + p] = Elem<DT>::narrow(v);
  }, [&](int q, float v) { ((T*)grad_bias)[(int64_t)e * d_out + q0 + q] = Elem<DT>::narrow(v); });
}

}  // namespace

hipError_t launch_expert_forward(const void* x, const void* w, const void* bias, const int32_t* offsets, int64_t rows,
                                 int d_in, int d_out, int E, bool bf16, int act, void* pre, void* out, hipStream_t stream) {
  const dim3 grid = grid_of_blocks((uint64_t)most_row_tiles(rows, E, kTile) * ((d_out + kTile - 1) / kTile));
  if (bf16)
    forward_kernel<BF16><<<grid, 256, 0, stream>>>(x, w, bias, offsets, rows, d_in, d_out, E, act, pre, out);
  else
    forward_kernel<F32><<<grid, 256, 0, stream>>>(x, w, bias, offsets, rows, d_in, d_out, E, act, pre, out);
  return hipGetLastError();
}

hipError_t launch_expert_input_grad(const void* grad_out, const void* w, const int32_t* offsets, int64_t rows, int d_in,
                                    int d_out, int E, bool bf16, int act, const void* pre, void* grad_x, hipStream_t stream) {
  const dim3 grid = grid_of_blocks((uint64_t)most_row_tiles(rows, E, kTile) * ((d_in + kTile - 1) / kTile));
  if (bf16)
    input_grad_kernel<BF16><<<grid, 256, 0, stream>>>(grad_out, w, offsets, rows, d_in, d_out, E, act, pre, grad_x);
  else
    input_grad_kernel<F32><<<grid, 256, 0, stream>>>(grad_out, w, offsets, rows, d_in, d_out, E, act, pre, grad_x);
  return hipGetLastError();
}

size_t expert_workspace_bytes(int64_t, int, int, int, bool) { return 0; }

hipError_t launch_expert_weight_grad(const void* grad_out, const void* x, const int32_t* offsets, int64_t rows, int d_in,
                                     int d_out, int E, bool bf16, void* grad_w, void* grad_bias, char*, hipStream_t stream) {
  const dim3 grid = grid_of_blocks((uint64_t)E * ((d_in + kTile - 1) / kTile) * ((d_out + kTile - 1) / kTile));
  if (bf16)
    weight_grad_kernel<BF16><<<grid, 256, 0, stream>>>(grad_out, x, offsets, rows, d_in, d_out, grad_w, grad_bias);
  else
    weight_grad_kernel<F32><<<grid, 256, 0, stream>>>(grad_out, x, offsets, rows, d_in, d_out, grad_w, grad_bias);
  return hipGetLastError();
}

}  // namespace lshmoe
