// Host-side error paths of the router's, the experts' and the 4-bit rows' entry points, for a build with AddressSanitizer and
// UndefinedBehaviorSanitizer on the host code of the checks (no GPU is touched: every call is rejected by them).
#include <limits.h>
#include <stdio.h>

#include "../../include/lshmoe.h"

static int failures = 0;
#define EXPECT(call, want)                                                                 \
  do {                                                                                     \
    const int got_ = (int)(call);                                                          \
    if (got_ != (int)(want)) {                                                             \
      printf("FAIL %s: got %s (%s)\n", #call, lshmoe_status_string(got_), lshmoe_last_error()); \
      ++failures;                                                                          \
    }                                                                                      \
  } while (0)

int main() {
  void* p = (void*)0x1000;   // never dereferenced
  void* odd = (void*)0x1008;
  int32_t *pi = (int32_t*)p, *oddi = (int32_t*)odd;
  float *pf = (float*)p, *oddf = (float*)odd;
  uint8_t *pb = (uint8_t*)p, *oddb = (uint8_t*)odd;
  const int64_t many = (int64_t)1 << 30;
  const uint32_t full = LSHMOE_FLAG_GATE_FULL_SOFTMAX;
  size_t bytes = 0;

  EXPECT(lshmoe_gate_topk(nullptr, 4, 8, 2, 0, pi, pf, nullptr), LSHMOE_ERR_NULL);
  EXPECT(lshmoe_gate_topk(pf, 4, 8, 2, 0, nullptr, pf, nullptr), LSHMOE_ERR_NULL);
  EXPECT(lshmoe_gate_topk(pf, 4, 8, 2, 0, pi, nullptr, nullptr), LSHMOE_ERR_NULL);
  EXPECT(lshmoe_gate_topk(pf, 0, 8, 2, 0, pi, pf, nullptr), LSHMOE_ERR_SHAPE);
  EXPECT(lshmoe_gate_topk(pf, LLONG_MIN, 8, 2, 0, pi, pf, nullptr), LSHMOE_ERR_SHAPE);
  EXPECT(lshmoe_gate_topk(pf, 4, INT_MIN, 2, 0, pi, pf, nullptr), LSHMOE_ERR_SHAPE);
  EXPECT(lshmoe_gate_topk(pf, 4, 8, 0, 0, pi, pf, nullptr), LSHMOE_ERR_SHAPE);
  EXPECT(lshmoe_gate_topk(pf, 4, 8, 9, 0, pi, pf, nullptr), LSHMOE_ERR_SHAPE);
  EXPECT(lshmoe_gate_topk(pf, many, 8, 2, 0, pi, pf, nullptr), LSHMOE_ERR_UNSUPPORTED);
  EXPECT(lshmoe_gate_topk(pf, LLONG_MAX, 8, 2, 0, pi, pf, nullptr), LSHMOE_ERR_UNSUPPORTED);
  EXPECT(lshmoe_gate_topk(pf, 4, 1025, 2, 0, pi, pf, nullptr), LSHMOE_ERR_UNSUPPORTED);
  EXPECT(lshmoe_gate_topk(pf, 4, INT_MAX, 2, 0, pi, pf, nullptr), LSHMOE_ERR_UNSUPPORTED);
  EXPECT(lshmoe_gate_topk(pf, 4, 1024, 65, 0, pi, pf, nullptr), LSHMOE_ERR_UNSUPPORTED);
  EXPECT(lshmoe_gate_topk(pf, 4, 8, 2, 1, pi, pf, nullptr), LSHMOE_ERR_UNSUPPORTED);
  EXPECT(lshmoe_gate_topk(oddf, 4, 8, 2, 0, pi, pf, nullptr), LSHMOE_ERR_UNSUPPORTED);
  EXPECT(lshmoe_gate_topk(pf, 4, 8, 2, 0, oddi, pf, nullptr), LSHMOE_ERR_UNSUPPORTED);
  EXPECT(lshmoe_gate_topk(pf, 4, 8, 2, 0, pi, oddf, nullptr), LSHMOE_ERR_UNSUPPORTED);
  EXPECT(lshmoe_gate_topk_backward(nullptr, pi, pf, pf, 4, 8, 2, full, pf, nullptr), LSHMOE_ERR_NULL);
  EXPECT(lshmoe_gate_topk_backward(pf, nullptr, pf, pf, 4, 8, 2, 0, pf, nullptr), LSHMOE_ERR_NULL);
  EXPECT(lshmoe_gate_topk_backward(pf, pi, pf, pf, 4, 8, 2, 0, nullptr, nullptr), LSHMOE_ERR_NULL);
  EXPECT(lshmoe_gate_topk_backward(nullptr, pi, pf, pf, 4, 8, 9, 0, pf, nullptr), LSHMOE_ERR_SHAPE);
  EXPECT(lshmoe_gate_topk_backward(nullptr, pi, pf, pf, 4, 8, 2, 4, pf, nullptr), LSHMOE_ERR_UNSUPPORTED);
  EXPECT(lshmoe_gate_topk_backward(nullptr, pi, pf, pf, 4, 8, 2, 0, oddf, nullptr), LSHMOE_ERR_UNSUPPORTED);

  for (lshmoe_dtype dt : {LSHMOE_F32, LSHMOE_BF16}) {
    auto forward = [&](const void* x, const void* w, const void* b, const int32_t* off, int64_t rows, int d_in, int d_out, int E,
                       int act, void* pre, void* out) {
      return lshmoe_expert_forward(x, w, b, off, rows, d_in, d_out, E, dt, (lshmoe_activation)act, pre, out, nullptr);
    };
    EXPECT(forward(nullptr, p, p, pi, 8, 64, 64, 2, 0, p, p), LSHMOE_ERR_NULL);
    EXPECT(forward(p, nullptr, p, pi, 8, 64, 64, 2, 0, p, p), LSHMOE_ERR_NULL);
    EXPECT(forward(p, p, p, nullptr, 8, 64, 64, 2, 0, p, p), LSHMOE_ERR_NULL);
    EXPECT(forward(p, p, p, pi, 8, 64, 64, 2, 0, p, nullptr), LSHMOE_ERR_NULL);
    EXPECT(forward(p, p, p, pi, 0, 64, 64, 2, 0, p, p), LSHMOE_ERR_SHAPE);
    EXPECT(forward(p, p, p, pi, LLONG_MIN, 64, 64, 2, 0, p, p), LSHMOE_ERR_SHAPE);
    EXPECT(forward(p, p, p, pi, 8, -64, 64, 2, 0, p, p), LSHMOE_ERR_SHAPE);
    EXPECT(forward(p, p, p, pi, 8, 64, 0, 2, 0, p, p), LSHMOE_ERR_SHAPE);
    EXPECT(forward(p, p, p, pi, 8, 64, 64, INT_MIN, 0, p, p), LSHMOE_ERR_SHAPE);
    EXPECT(forward(p, p, p, pi, 8, 63, 64, 2, 0, p, p), LSHMOE_ERR_UNSUPPORTED);
    EXPECT(forward(p, p, p, pi, 8, 64, 66, 2, 0, p, p), LSHMOE_ERR_UNSUPPORTED);
    EXPECT(forward(p, p, p, pi, 8, INT_MAX, 64, 2, 0, p, p), LSHMOE_ERR_UNSUPPORTED);
    EXPECT(forward(p, p, p, pi, 8, 64, 1 << 23, 2, 0, p, p), LSHMOE_ERR_UNSUPPORTED);          // rows of 8 MiB and more
    EXPECT(forward(p, p, p, pi, 8, 1 << 20, 1 << 20, 2, 0, p, p), LSHMOE_ERR_UNSUPPORTED);     // 2 GiB for an expert and more
    EXPECT(forward(p, p, p, pi, 8, 64, 64, 4097, 0, p, p), LSHMOE_ERR_UNSUPPORTED);
    EXPECT(forward(p, p, p, pi, many, 64, 64, 2, 0, p, p), LSHMOE_ERR_UNSUPPORTED);
    EXPECT(forward(p, p, p, pi, LLONG_MAX, 64, 64, 2, 0, p, p), LSHMOE_ERR_UNSUPPORTED);
    EXPECT(forward(p, p, p, pi, many - 1, 64, 4096, 2, 0, p, p), LSHMOE_ERR_UNSUPPORTED);      // too many bytes of rows
    EXPECT(forward(p, p, p, pi, 8, 64, 64, 2, 3, p, p), LSHMOE_ERR_UNSUPPORTED);
    EXPECT(forward(p, p, p, pi, 8, 64, 64, 2, -1, p, p), LSHMOE_ERR_UNSUPPORTED);
    EXPECT(forward(odd, p, p, pi, 8, 64, 64, 2, 0, p, p), LSHMOE_ERR_UNSUPPORTED);
    EXPECT(forward(p, odd, p, pi, 8, 64, 64, 2, 0, p, p), LSHMOE_ERR_UNSUPPORTED);
    EXPECT(forward(p, p, odd, pi, 8, 64, 64, 2, 0, p, p), LSHMOE_ERR_UNSUPPORTED);
    EXPECT(forward(p, p, p, oddi, 8, 64, 64, 2, 0, p, p), LSHMOE_ERR_UNSUPPORTED);
    EXPECT(forward(p, p, p, pi, 8, 64, 64, 2, 0, odd, p), LSHMOE_ERR_UNSUPPORTED);
    EXPECT(forward(p, p, p, pi, 8, 64, 64, 2, 0, p, odd), LSHMOE_ERR_UNSUPPORTED);
    EXPECT(lshmoe_expert_backward_input(p, p, pi, 8, 64, 64, 2, dt, LSHMOE_ACT_GELU, nullptr, p, nullptr), LSHMOE_ERR_NULL);
    EXPECT(lshmoe_expert_backward_input(p, p, pi, 8, 64, 64, 2, dt, LSHMOE_ACT_NONE, nullptr, nullptr, nullptr), LSHMOE_ERR_NULL);
    EXPECT(lshmoe_expert_backward_input(p, p, pi, 8, 64, 64, 2, dt, LSHMOE_ACT_RELU, odd, p, nullptr), LSHMOE_ERR_UNSUPPORTED);
    EXPECT(lshmoe_expert_backward_input(p, p, pi, 8, 64, 62, 2, dt, LSHMOE_ACT_NONE, nullptr, p, nullptr), LSHMOE_ERR_UNSUPPORTED);
    EXPECT(lshmoe_expert_workspace_bytes(8, 64, 64, 2, dt, nullptr), LSHMOE_ERR_NULL);
    EXPECT(lshmoe_expert_workspace_bytes(8, 0, 64, 2, dt, &bytes), LSHMOE_ERR_SHAPE);
    EXPECT(lshmoe_expert_workspace_bytes(many, 64, 64, 2, dt, &bytes), LSHMOE_ERR_UNSUPPORTED);
    EXPECT(lshmoe_expert_workspace_bytes(5000, 256, 256, 2, dt, &bytes), LSHMOE_OK);
    if (bytes == 0) { printf("FAIL no workspace where experts may be cut\n"); ++failures; }
    EXPECT(lshmoe_expert_backward_weight(p, p, pi, 5000, 256, 256, 2, dt, p, nullptr, nullptr, bytes, nullptr), LSHMOE_ERR_WORKSPACE);
    EXPECT(lshmoe_expert_backward_weight(p, p, pi, 5000, 256, 256, 2, dt, p, nullptr, (void*)0x1010, bytes, nullptr), LSHMOE_ERR_WORKSPACE);
    EXPECT(lshmoe_expert_backward_weight(p, p, pi, 5000, 256, 256, 2, dt, p, nullptr, p, bytes - 1, nullptr), LSHMOE_ERR_WORKSPACE);
    EXPECT(lshmoe_expert_backward_weight(p, p, pi, 5000, 256, 256, 2, dt, nullptr, p, p, bytes, nullptr), LSHMOE_ERR_NULL);
    EXPECT(lshmoe_expert_backward_weight(p, p, pi, 5000, 256, 256, 2, dt, p, odd, p, bytes, nullptr), LSHMOE_ERR_UNSUPPORTED);

    EXPECT(lshmoe_mx4_quantize(nullptr, 4, 64, dt, pb, pb, nullptr), LSHMOE_ERR_NULL);
    EXPECT(lshmoe_mx4_quantize(p, 4, 64, dt, pb, nullptr, nullptr), LSHMOE_ERR_NULL);
    EXPECT(lshmoe_mx4_quantize(p, 4, 0, dt, pb, pb, nullptr), LSHMOE_ERR_SHAPE);
    EXPECT(lshmoe_mx4_quantize(p, -4, 64, dt, pb, pb, nullptr), LSHMOE_ERR_SHAPE);
    EXPECT(lshmoe_mx4_quantize(p, 4, 48, dt, pb, pb, nullptr), LSHMOE_ERR_UNSUPPORTED);
    EXPECT(lshmoe_mx4_quantize(p, many, 64, dt, pb, pb, nullptr), LSHMOE_ERR_UNSUPPORTED);
    EXPECT(lshmoe_mx4_quantize(p, 4, 64, dt, pb, oddb, nullptr), LSHMOE_ERR_UNSUPPORTED);
    EXPECT(lshmoe_mx4_dequantize(pb, pb, 4, 64, dt, nullptr, nullptr), LSHMOE_ERR_NULL);
    EXPECT(lshmoe_mx4_dequantize(pb, pb, 4, 40, dt, p, nullptr), LSHMOE_ERR_UNSUPPORTED);
    EXPECT(lshmoe_mx4_dequantize(oddb, pb, 4, 64, dt, p, nullptr), LSHMOE_ERR_UNSUPPORTED);
    auto forward4 = [&](const uint8_t* xs, const uint8_t* ws, int d_in, int d_out, int act, void* out) {
      return lshmoe_expert_forward_mx4(pb, xs, pb, ws, nullptr, pi, 8, d_in, d_out, 2, dt, (lshmoe_activation)act, out, nullptr);
    };
    EXPECT(forward4(nullptr, pb, 64, 64, 0, p), LSHMOE_ERR_NULL);
    EXPECT(forward4(pb, nullptr, 64, 64, 0, p), LSHMOE_ERR_NULL);
    EXPECT(forward4(pb, pb, 64, 64, 0, nullptr), LSHMOE_ERR_NULL);
    EXPECT(forward4(pb, pb, 0, 64, 0, p), LSHMOE_ERR_SHAPE);
    EXPECT(forward4(pb, pb, 48, 64, 0, p), LSHMOE_ERR_UNSUPPORTED);
    EXPECT(forward4(pb, pb, 64, 62, 0, p), LSHMOE_ERR_UNSUPPORTED);
    EXPECT(forward4(pb, pb, 64, 64, 9, p), LSHMOE_ERR_UNSUPPORTED);
    EXPECT(forward4(oddb, pb, 64, 64, 0, p), LSHMOE_ERR_UNSUPPORTED);
    EXPECT(forward4(pb, pb, 64, 64, 0, odd), LSHMOE_ERR_UNSUPPORTED);
  }
  EXPECT(lshmoe_expert_forward(p, p, p, pi, 8, 64, 64, 2, (lshmoe_dtype)7, LSHMOE_ACT_NONE, p, p, nullptr), LSHMOE_ERR_UNSUPPORTED);
  EXPECT(lshmoe_mx4_quantize(p, 4, 64, (lshmoe_dtype)7, pb, pb, nullptr), LSHMOE_ERR_UNSUPPORTED);
  EXPECT(lshmoe_expert_workspace_bytes(8, 64, 64, 2, (lshmoe_dtype)-1, &bytes), LSHMOE_ERR_UNSUPPORTED);
  printf("%d failures\n", failures);
  return failures ? 1 : 0;
}
