// C ABI of the router, the experts' products and the 4-bit rows: argument checks on the host, then kernel launches.  As in
// api.hip every check runs before the first HIP call.
#include <initializer_list>

#include "api.h"
#include "kernels.h"

namespace {

using lshmoe::check_row;
using lshmoe::fail;
using lshmoe::hip_fail;
using lshmoe::item_size;
using lshmoe::kMaxAssignments;
using lshmoe::ok;

constexpr int kMaxProductExperts = 4096;

// The kernels move 16-byte pieces.
lshmoe_status check_aligned(std::initializer_list<const void*> pointers) {
  for (const void* p : pointers)
    if (((uintptr_t)p & 15u) != 0) return fail(LSHMOE_ERR_UNSUPPORTED, "pointer %p is not 16-byte aligned", p);
  return LSHMOE_OK;
}

lshmoe_status check_gate(int64_t T, int E, int k, uint32_t flags) {
  if (T <= 0 || E <= 0 || k <= 0)
    return fail(LSHMOE_ERR_SHAPE, "T, E, k must be positive (T=%lld, E=%d, k=%d)", (long long)T, E, k);
  if (k > E) return fail(LSHMOE_ERR_SHAPE, "k=%d experts per token exceeds E=%d experts", k, E);
  if (T >= kMaxAssignments) return fail(LSHMOE_ERR_UNSUPPORTED, "T = %lld tokens; the limit is 2^30 - 1", (long long)T);
  if (E > lshmoe::kMaxGateExperts || k > lshmoe::kMaxGateChoices)
    return fail(LSHMOE_ERR_UNSUPPORTED, "E=%d, k=%d; the limits are %d experts and %d of them for a token", E, k,
                lshmoe::kMaxGateExperts, lshmoe::kMaxGateChoices);
  if (flags & ~(uint32_t)LSHMOE_FLAG_GATE_FULL_SOFTMAX) return fail(LSHMOE_ERR_UNSUPPORTED, "unknown flag bits 0x%x", flags);
  return LSHMOE_OK;
}

// rows x d in dtype, as every entry point that moves rows takes them
lshmoe_status check_rows(int64_t rows, int d, int dt) {
  if (lshmoe_status st = check_row(d, dt)) return st;
  if (rows >= kMaxAssignments) return fail(LSHMOE_ERR_UNSUPPORTED, "%lld rows; the limit is 2^30 - 1", (long long)rows);
  if ((uint64_t)rows * ((size_t)d * item_size(dt) / 16) > 0xffffff00ull)
    return fail(LSHMOE_ERR_UNSUPPORTED, "rows * d is too large for one launch");
  return LSHMOE_OK;
}

lshmoe_status check_product(int64_t rows, int d_in, int d_out, int E, int dt) {
  if (rows <= 0 || d_in <= 0 || d_out <= 0 || E <= 0)
    return fail(LSHMOE_ERR_SHAPE, "rows, d_in, d_out, E must be positive (rows=%lld, d_in=%d, d_out=%d, E=%d)",
                (long long)rows, d_in, d_out, E);
  for (int d : {d_in, d_out}) {
    if (lshmoe_status st = check_rows(rows, d, dt)) return st;
    if ((size_t)d * item_size(dt) >= (size_t)8 << 20) return fail(LSHMOE_ERR_UNSUPPORTED, "rows of %d elements are too long", d);
  }
  if (E > kMaxProductExperts) return fail(LSHMOE_ERR_UNSUPPORTED, "E = %d experts; the limit is %d", E, kMaxProductExperts);
  if ((uint64_t)d_in * d_out * item_size(dt) >= 1ull << 31)
    return fail(LSHMOE_ERR_UNSUPPORTED, "one expert's %d x %d weights are 2 GiB or more", d_out, d_in);
  return LSHMOE_OK;
}

lshmoe_status check_activation(int act) {
  if (act != LSHMOE_ACT_NONE && act != LSHMOE_ACT_RELU && act != LSHMOE_ACT_GELU)
    return fail(LSHMOE_ERR_UNSUPPORTED, "unknown activation %d", act);
  return LSHMOE_OK;
}

lshmoe_status check_mx4(int64_t rows, int d, int dt) {
  if (rows <= 0 || d <= 0) return fail(LSHMOE_ERR_SHAPE, "rows and d must be positive (rows=%lld, d=%d)", (long long)rows, d);
  if (lshmoe_status st = check_rows(rows, d, dt)) return st;
  if (d % 32 != 0) return fail(LSHMOE_ERR_UNSUPPORTED, "d = %d is not a multiple of the 32 numbers of a block", d);
  return LSHMOE_OK;
}

}  // namespace

extern "C" {

lshmoe_status lshmoe_gate_topk(const float* logits, int64_t T, int32_t E, int32_t k, uint32_t flags, int32_t* expert,
                               float* gate_weight, void* stream) {
  if (!logits || !expert || !gate_weight) return fail(LSHMOE_ERR_NULL, "logits, expert and gate_weight must be non-NULL");
  if (lshmoe_status st = check_gate(T, E, k, flags)) return st;
  if (lshmoe_status st = check_aligned({logits, expert, gate_weight})) return st;
  hipError_t e = lshmoe::launch_gate_topk(logits, T, E, k, (flags & LSHMOE_FLAG_GATE_FULL_SOFTMAX) != 0, expert, gate_weight,
                                          (hipStream_t)stream);
  if (e != hipSuccess) return hip_fail("gate top-k launch", e);
  return ok();
}

lshmoe_status lshmoe_gate_topk_backward(const float* logits, const int32_t* expert, const float* gate_weight,
                                        const float* grad_gate_weight, int64_t T, int32_t E, int32_t k, uint32_t flags,
                                        float* grad_logits, void* stream) {
  if (!expert || !gate_weight || !grad_gate_weight || !grad_logits)
    return fail(LSHMOE_ERR_NULL, "an input or output pointer is NULL");
  if (lshmoe_status st = check_gate(T, E, k, flags)) return st;
  const bool full = (flags & LSHMOE_FLAG_GATE_FULL_SOFTMAX) != 0;
  if (full && !logits) return fail(LSHMOE_ERR_NULL, "logits are required with LSHMOE_FLAG_GATE_FULL_SOFTMAX");
  if (lshmoe_status st = check_aligned({logits, expert, gate_weight, grad_gate_weight, grad_logits})) return st;
  hipError_t e = lshmoe::launch_gate_topk_backward(logits, expert, gate_weight, grad_gate_weight, T, E, k, full, grad_logits,
                                                   (hipStream_t)stream);
  if (e != hipSuccess) return hip_fail("gate top-k backward launch", e);
  return ok();
}

lshmoe_status lshmoe_expert_forward(const void* x, const void* w, const void* bias, const int32_t* expert_offsets,
                                    int64_t rows, int32_t d_in, int32_t d_out, int32_t E, lshmoe_dtype dtype,
                                    lshmoe_activation act, void* pre, void* out, void* stream) {
  if (!x || !w || !expert_offsets || !out) return fail(LSHMOE_ERR_NULL, "x, w, expert_offsets and out must be non-NULL");
  if (lshmoe_status st = check_product(rows, d_in, d_out, E, (int)dtype)) return st;
  if (lshmoe_status st = check_activation((int)act)) return st;
  if (lshmoe_status st = check_aligned({x, w, bias, expert_offsets, pre, out})) return st;
  hipError_t e = lshmoe::launch_expert_forward(x, w, bias, expert_offsets, rows, d_in, d_out, E, dtype == LSHMOE_BF16,
                                               (int)act, pre, out, (hipStream_t)stream);
  if (e != hipSuccess) return hip_fail("expert forward launch", e);
  return ok();
}

lshmoe_status lshmoe_expert_backward_input(const void* grad_out, const void* w, const int32_t* expert_offsets, int64_t rows,
                                           int32_t d_in, int32_t d_out, int32_t E, lshmoe_dtype dtype, lshmoe_activation act,
                                           const void* pre, void* grad_x, void* stream) {
  if (!grad_out || !w || !expert_offsets || !grad_x)
    return fail(LSHMOE_ERR_NULL, "grad_out, w, expert_offsets and grad_x must be non-NULL");
  if (lshmoe_status st = check_product(rows, d_in, d_out, E, (int)dtype)) return st;
  if (lshmoe_status st = check_activation((int)act)) return st;
  if (act != LSHMOE_ACT_NONE && !pre) return fail(LSHMOE_ERR_NULL, "pre is required with an activation");
  if (lshmoe_status st = check_aligned({grad_out, w, expert_offsets, pre, grad_x})) return st;
  hipError_t e = lshmoe::launch_expert_input_grad(grad_out, w, expert_offsets, rows, d_in, d_out, E, dtype == LSHMOE_BF16,
                                                  (int)act, pre, grad_x, (hipStream_t)stream);
  if (e != hipSuccess) return hip_fail("expert input gradient launch", e);
  return ok();
}

lshmoe_status lshmoe_expert_workspace_bytes(int64_t rows, int32_t d_in, int32_t d_out, int32_t E, lshmoe_dtype dtype,
                                            size_t* out_bytes) {
  if (!out_bytes) return fail(LSHMOE_ERR_NULL, "out_bytes is NULL");
  if (lshmoe_status st = check_product(rows, d_in, d_out, E, (int)dtype)) return st;
  *out_bytes = lshmoe::expert_workspace_bytes(rows, d_in, d_out, dtype == LSHMOE_BF16);
  return ok();
}

lshmoe_status lshmoe_expert_backward_weight(const void* grad_out, const void* x, const int32_t* expert_offsets, int64_t rows,
                                            int32_t d_in, int32_t d_out, int32_t E, lshmoe_dtype dtype, void* grad_w,
                                            void* grad_bias, void* workspace, size_t workspace_bytes, void* stream) {
  if (!grad_out || !x || !expert_offsets || !grad_w)
    return fail(LSHMOE_ERR_NULL, "grad_out, x, expert_offsets and grad_w must be non-NULL");
  if (lshmoe_status st = check_product(rows, d_in, d_out, E, (int)dtype)) return st;
  if (lshmoe_status st = check_aligned({grad_out, x, expert_offsets, grad_w, grad_bias})) return st;
  const size_t need = lshmoe::expert_workspace_bytes(rows, d_in, d_out, dtype == LSHMOE_BF16);
  if (need > 0) {
    if (!workspace) return fail(LSHMOE_ERR_WORKSPACE, "workspace is NULL (%zu bytes needed)", need);
    if (((uintptr_t)workspace & 255u) != 0) return fail(LSHMOE_ERR_WORKSPACE, "workspace is not 256-byte aligned");
    if (workspace_bytes < need) return fail(LSHMOE_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, need);
  }
  hipError_t e = lshmoe::launch_expert_weight_grad(grad_out, x, expert_offsets, rows, d_in, d_out, E, dtype == LSHMOE_BF16,
                                                   grad_w, grad_bias, (char*)workspace, (hipStream_t)stream);
  if (e != hipSuccess) return hip_fail("expert weight gradient launch", e);
  return ok();
}

lshmoe_status lshmoe_mx4_quantize(const void* x, int64_t rows, int32_t d, lshmoe_dtype dtype, uint8_t* codes, uint8_t* scales,
                                  void* stream) {
  if (!x || !codes || !scales) return fail(LSHMOE_ERR_NULL, "x, codes and scales must be non-NULL");
  if (lshmoe_status st = check_mx4(rows, d, (int)dtype)) return st;
  if (lshmoe_status st = check_aligned({x, codes, scales})) return st;
  hipError_t e = lshmoe::launch_mx4_quantize(x, rows, d, dtype == LSHMOE_BF16, codes, scales, (hipStream_t)stream);
  if (e != hipSuccess) return hip_fail("4-bit quantisation launch", e);
  return ok();
}

lshmoe_status lshmoe_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int32_t d, lshmoe_dtype dtype,
                                    void* out, void* stream) {
  if (!codes || !scales || !out) return fail(LSHMOE_ERR_NULL, "codes, scales and out must be non-NULL");
  if (lshmoe_status st = check_mx4(rows, d, (int)dtype)) return st;
  if (lshmoe_status st = check_aligned({codes, scales, out})) return st;
  hipError_t e = lshmoe::launch_mx4_dequantize(codes, scales, rows, d, dtype == LSHMOE_BF16, out, (hipStream_t)stream);
  if (e != hipSuccess) return hip_fail("4-bit read-back launch", e);
  return ok();
}

lshmoe_status lshmoe_expert_forward_mx4(const uint8_t* x_codes, const uint8_t* x_scales, const uint8_t* w_codes,
                                        const uint8_t* w_scales, const void* bias, const int32_t* expert_offsets,
                                        int64_t rows, int32_t d_in, int32_t d_out, int32_t E, lshmoe_dtype dtype,
                                        lshmoe_activation act, void* out, void* stream) {
  if (!x_codes || !x_scales || !w_codes || !w_scales || !expert_offsets || !out)
    return fail(LSHMOE_ERR_NULL, "an input or output pointer is NULL");
  if (lshmoe_status st = check_product(rows, d_in, d_out, E, (int)dtype)) return st;
  if (d_in % 32 != 0) return fail(LSHMOE_ERR_UNSUPPORTED, "d_in = %d is not a multiple of the 32 numbers of a block", d_in);
  if (lshmoe_status st = check_activation((int)act)) return st;
  if (lshmoe_status st = check_aligned({x_codes, x_scales, w_codes, w_scales, bias, expert_offsets, out})) return st;
  hipError_t e = lshmoe::launch_expert_forward_mx4(x_codes, x_scales, w_codes, w_scales, bias, expert_offsets, rows, d_in, d_out,
                                                   E, dtype == LSHMOE_BF16, (int)act, out, (hipStream_t)stream);
  if (e != hipSuccess) return hip_fail("expert 4-bit forward launch", e);
  return ok();
}

}  // extern "C"
