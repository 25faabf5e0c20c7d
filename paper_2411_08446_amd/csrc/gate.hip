// Router: the k experts of a token from the logits of its gate, with their weights, and the gradient of the logits.
//
// G lanes share a token (G a power of two, up to C = 4 pieces of 4 logits to a lane, c = 0 .. C - 1); lane i of them holds the logits
// 4 (i + G c) + j, so that a token's row comes in whole 16-byte pieces.  Choosing is k rounds of an arg-max over the lanes' own best candidates: the
// comparison is on (value, lower index), so a round's winner does not depend on the order of the exchanges.
//
// The floor is the read of the logits (and in the backward pass the write of their gradient): 4 E bytes per token.  65536 tokens of 64
// experts, k = 2: 8.8 us, 8.0 backward with the softmax over all; k rounds of exchanges are a chain that a lane waits for (k = 8 of 256
// experts: 38 us, 1.8 TB/s), hence 16 lanes to a token, whose exchanges stay within the vector unit (64 lanes: 106 us).
#include <type_traits>

#include "kernels.h"

namespace lshmoe {

namespace {

constexpr int kGateThreads = 256;

// Ascending order of the floats as unsigned integers: -0 and +0 are one value, NaN is above everything.  0 is below every
// value's number and marks a logit that is taken or not there.
__device__ __forceinline__ uint32_t order_of(float v) {
  if (v != v) return 0xffffffffu;
  const uint32_t u = __float_as_uint(v + 0.0f);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// f(std::integral_constant<int, M>) for M = 1, 2, .. below G.
template <int G, int M = 1, typename F> __device__ __forceinline__ void over_halves(F&& f) {
  if constexpr (M < G) {
    f(std::integral_constant<int, M>{});
    over_halves<G, 2 * M>(f);
  }
}

template <int G> __device__ __forceinline__ float group_sum(float v) {
  over_halves<G>([&](auto m) { v += other_half<decltype(m)::value>(v); });
  return v;
}

// The larger one; a NaN stays one.
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }

template <int G> __device__ __forceinline__ float group_max(float v) {
  over_halves<G>([&](auto m) { v = larger(v, other_half<decltype(m)::value>(v)); });
  return v;
}

// A lane's logits; what lies behind the row is -inf.
template <int G, int C, bool VEC>
__device__ __forceinline__ void load_logits(const float* __restrict__ row, int lane, int E, float (&v)[4 * C]) {
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int e0 = 4 * (lane + G * c);
    if (VEC) {
      float4 q = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
      if (e0 < E) q = *reinterpret_cast<const float4*>(row + e0);
      v[4 * c] = q.x; v[4 * c + 1] = q.y; v[4 * c + 2] = q.z; v[4 * c + 3] = q.w;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[4 * c + j] = e0 + j < E ? row[e0 + j] : -INFINITY;
    }
  }
}

// G lanes to a token, C pieces of 4 logits to a lane.  VEC: rows of whole pieces.
template <int G, int C, bool VEC>
__global__ __launch_bounds__(kGateThreads) void gate_topk_kernel(const float* __restrict__ logits, uint32_t T, int E, int k,
                                                                 bool full, int32_t* __restrict__ expert,
                                                                 float* __restrict__ weight) {
  constexpr int kTokens = kGateThreads / G;
  __shared__ float chosen[kTokens * (G * C < 16 ? 4 * G * C : 64)];   // k <= 64 and k <= E
  const int lane = (int)threadIdx.x % G, slot = (int)threadIdx.x / G;
  const uint64_t t = linear_block() * kTokens + slot;
  const bool live = t < T;
  float v[4 * C];
  load_logits<G, C, VEC>(logits + (live ? t : 0) * (uint64_t)E, lane, E, v);
  uint32_t left[4 * C];                       // order of what is left to choose from
#pragma unroll
  for (int i = 0; i < 4 * C; ++i) left[i] = 4 * (lane + G * (i / 4)) + i % 4 < E ? order_of(v[i]) : 0u;
  float top = 0.0f, sum = 0.0f;
  for (int j = 0; j < k; ++j) {
    uint32_t best = left[0];
    int at = 4 * lane;
    float val = v[0];
#pragma unroll
    for (int i = 1; i < 4 * C; ++i) {
      if (left[i] > best) {                   // ascending index: the lowest of equal values stays
        best = left[i];
        at = 4 * (lane + G * (i / 4)) + i % 4;
        val = v[i];
      }
    }
    over_halves<G>([&](auto m) {
      constexpr int M = decltype(m)::value;
      const uint32_t obest = other_half<M>(best), oat = other_half<M>((uint32_t)at);
      const float oval = other_half<M>(val);
      if (obest > best || (obest == best && (int)oat < at)) {
        best = obest;
        at = (int)oat;
        val = oval;
      }
    });
#pragma unroll
    for (int i = 0; i < 4 * C; ++i)
      if (4 * (lane + G * (i / 4)) + i % 4 == at) left[i] = 0u;
    if (j == 0) top = val;
    sum += expf(val - top);
    if (lane == 0) {
      chosen[slot * k + j] = val;
      if (live) expert[t * (uint64_t)k + j] = at;
    }
  }
  if (full) {
    float part = 0.0f;
#pragma unroll
    for (int i = 0; i < 4 * C; ++i) part += expf(v[i] - top);
    sum = group_sum<G>(part);
  }
  __syncthreads();
  if (!live) return;
  // a token all of whose experts are masked has no weight to give
  for (int j = lane; j < k; j += G)
    weight[t * (uint64_t)k + j] = top == -INFINITY ? 0.0f : expf(chosen[slot * k + j] - top) / sum;
}

// dL/dlogits.  Over the chosen experts (w the weights, g = dL/dw):  w_j (g_j - <w, g>) at the chosen ones, 0 elsewhere.  Over
// all experts (p the softmax):  p_e ([e chosen] g_e - <w, g>).
template <int G, int C, bool VEC>
__global__ __launch_bounds__(kGateThreads) void gate_topk_backward_kernel(const float* __restrict__ logits,
                                                                          const int32_t* __restrict__ expert,
                                                                          const float* __restrict__ weight,
                                                                          const float* __restrict__ grad_weight, uint32_t T,
                                                                          int E, int k, bool full,
                                                                          float* __restrict__ grad_logits) {
  constexpr int kTokens = kGateThreads / G;
  const int lane = (int)threadIdx.x % G, slot = (int)threadIdx.x / G;
  const uint64_t t = linear_block() * kTokens + slot;
  const bool live = t < T;
  const uint64_t a0 = (live ? t : 0) * (uint64_t)k;
  float v[4 * C];
  if (full) load_logits<G, C, VEC>(logits + (live ? t : 0) * (uint64_t)E, lane, E, v);
  float mean = 0.0f;
  bool any = false;        // a token all of whose experts are masked has only weights of 0 (the largest logit's is 1 / E at least)
  for (int j = 0; j < k; ++j) {
    mean = fmaf(weight[a0 + j], grad_weight[a0 + j], mean);
    any |= weight[a0 + j] != 0.0f;
  }
  float out[4 * C] = {};
  for (int j = 0; j < k; ++j) {
    const int e = min((uint32_t)expert[a0 + j], (uint32_t)(E - 1));
    const float g = grad_weight[a0 + j];
    // (whatever the gradients of its weights are: behind a masked token there may be rows that hold anything)
    const float term = full ? g : any ? weight[a0 + j] * (g - mean) : 0.0f;
#pragma unroll
    for (int i = 0; i < 4 * C; ++i)
      if (4 * (lane + G * (i / 4)) + i % 4 == e) out[i] += term;
  }
  if (full) {
    float top = v[0], sum = 0.0f;
#pragma unroll
    for (int i = 1; i < 4 * C; ++i) top = larger(top, v[i]);
    top = group_max<G>(top);
#pragma unroll
    for (int i = 0; i < 4 * C; ++i) {
      v[i] = expf(v[i] - top);
      sum += v[i];
    }
    sum = group_sum<G>(sum);
#pragma unroll
    for (int i = 0; i < 4 * C; ++i) out[i] = top == -INFINITY ? 0.0f : v[i] / sum * (out[i] - mean);
  }
  if (!live) return;
  float* row = grad_logits + t * (uint64_t)E;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int e0 = 4 * (lane + G * c);
    if (VEC) {
      if (e0 < E) *reinterpret_cast<float4*>(row + e0) = make_float4(out[4 * c], out[4 * c + 1], out[4 * c + 2], out[4 * c + 3]);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (e0 + j < E) row[e0 + j] = out[4 * c + j];
    }
  }
}

template <int G, int C> hipError_t launch_topk(const float* logits, int64_t T, int E, int k, bool full, int32_t* expert,
                                               float* weight, hipStream_t stream) {
  const dim3 grid = grid_of_blocks(((uint64_t)T + kGateThreads / G - 1) / (kGateThreads / G));
  if (E % 4 == 0)
    gate_topk_kernel<G, C, true><<<grid, kGateThreads, 0, stream>>>(logits, (uint32_t)T, E, k, full, expert, weight);
  else
    gate_topk_kernel<G, C, false><<<grid, kGateThreads, 0, stream>>>(logits, (uint32_t)T, E, k, full, expert, weight);
  return hipGetLastError();
}

template <int G, int C> hipError_t launch_backward(const float* logits, const int32_t* expert, const float* weight,
                                                   const float* grad_weight, int64_t T, int E, int k, bool full,
                                                   float* grad_logits, hipStream_t stream) {
  const dim3 grid = grid_of_blocks(((uint64_t)T + kGateThreads / G - 1) / (kGateThreads / G));
  if (E % 4 == 0)
    gate_topk_backward_kernel<G, C, true><<<grid, kGateThreads, 0, stream>>>(logits, expert, weight, grad_weight, (uint32_t)T,
                                                                             E, k, full, grad_logits);
  else
    gate_topk_backward_kernel<G, C, false><<<grid, kGateThreads, 0, stream>>>(logits, expert, weight, grad_weight, (uint32_t)T,
                                                                              E, k, full, grad_logits);
  return hipGetLastError();
}

}  // namespace

#define LSHMOE_GATE_SHAPES(call)                   \
  if (E <= 4) return call(1, 1);                   \
  if (E <= 8) return call(2, 1);                   \
  if (E <= 16) return call(4, 1);                  \
  if (E <= 32) return call(8, 1);                  \
  if (E <= 64) return call(16, 1);                 \
  if (E <= 128) return call(16, 2);                \
  if (E <= 256) return call(16, 4);                \
  if (E <= 512) return call(32, 4);                \
  return call(64, 4);

hipError_t launch_gate_topk(const float* logits, int64_t T, int E, int k, bool full, int32_t* expert, float* weight,
                            hipStream_t stream) {
#define CALL(G, C) launch_topk<G, C>(logits, T, E, k, full, expert, weight, stream)
  LSHMOE_GATE_SHAPES(CALL)
#undef CALL
}

hipError_t launch_gate_topk_backward(const float* logits, const int32_t* expert, const float* weight,
                                     const float* grad_weight, int64_t T, int E, int k, bool full, float* grad_logits,
                                     hipStream_t stream) {
#define CALL(G, C) launch_backward<G, C>(logits, expert, weight, grad_weight, T, E, k, full, grad_logits, stream)
  LSHMOE_GATE_SHAPES(CALL)
#undef CALL
}

}  // namespace lshmoe
