// Records the launches that the router's, the experts' and the 4-bit rows' entry points make over their documented ranges.  The
// program defines the runtime's launch calls itself, so no GPU is needed and nothing is launched; pointers are never
// dereferenced.
//
// A dispatch counts the work-items of a dimension in 32 bits, a workgroup has at most 160 KB of LDS, and the products' tiles are
// shared out over grids of a multiple of 8 workgroups.
#include <hip/hip_runtime.h>
#include <stdio.h>

#include "../../include/lshmoe.h"

static int failures = 0, launches = 0;
static long long now_rows = 0;
static int now_E = 0, now_in = 0, now_out = 0;
static const char* now_call = "";
static size_t lds_asked = 0;
static dim3 push_grid, push_block;
static size_t push_lds;
static hipStream_t push_stream;

static void fail(const char* what) {
  if (++failures <= 20)
    printf("FAIL %s rows=%lld E=%d d_in=%d d_out=%d: %s\n", now_call, now_rows, now_E, now_in, now_out, what);
}

extern "C" {
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t stream) {
  push_grid = grid; push_block = block; push_lds = lds; push_stream = stream;
  return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* stream) {
  *grid = push_grid; *block = push_block; *lds = push_lds; *stream = push_stream;
  return hipSuccess;
}
hipError_t hipLaunchKernel(const void*, dim3 grid, dim3 block, void**, size_t lds, hipStream_t) {
  ++launches;
  const unsigned long long limit = 1ull << 32;
  if ((unsigned long long)grid.x * block.x >= limit || (unsigned long long)grid.y * block.y >= limit || grid.z != 1 ||
      grid.y > 65535u || grid.x == 0 || grid.y == 0)
    fail("grid out of range");
  if (lds > 160 * 1024 || lds > lds_asked) fail("more LDS than there is or than was asked for");
  if (lds > 0 && (grid.x % 8 != 0 || grid.y != 1)) fail("tiles' grid is no multiple of 8");
  lds_asked = 0;
  return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipFuncSetAttribute(const void*, hipFuncAttribute, int bytes) {
  lds_asked = (size_t)bytes;
  return hipSuccess;
}
}

static void expect_ok(int status) {
  if (status != LSHMOE_OK) fail(lshmoe_last_error());
}

int main() {
  void* p = (void*)0x1000;
  int32_t* pi = (int32_t*)p;
  float* pf = (float*)p;
  uint8_t* pb = (uint8_t*)p;
  const long long top = (1ll << 30) - 1;
  now_call = "gate";
  for (long long T : {1ll, 63ll, 257ll, 65536ll, 1ll << 27, (1ll << 29) + 1, top})
    for (int E : {1, 3, 4, 5, 8, 16, 17, 33, 64, 65, 128, 129, 256, 257, 512, 513, 1021, 1024})
      for (int k : {1, 2, 8, 64}) {
        if (k > E) continue;
        now_rows = T;
        now_E = E;
        for (uint32_t flags : {0u, (uint32_t)LSHMOE_FLAG_GATE_FULL_SOFTMAX}) {
          expect_ok(lshmoe_gate_topk(pf, T, E, k, flags, pi, pf, nullptr));
          expect_ok(lshmoe_gate_topk_backward(pf, pi, pf, pf, T, E, k, flags, pf, nullptr));
        }
      }
  for (lshmoe_dtype dtype : {LSHMOE_F32, LSHMOE_BF16}) {
    const int piece = dtype == LSHMOE_BF16 ? 8 : 4;
    const unsigned long long item = 16 / piece;
    for (long long rows : {1ll, 8ll, 74ll, 512ll, 513ll, 4096ll, 16385ll, 131072ll, 1ll << 20, 1ll << 26, top})
      for (int E : {1, 8, 64, 65, 4096})
        for (int d_in : {piece, 32, 72, 768, 4096, 32768, (8 << 20) / (int)item - piece})
          for (int d_out : {piece, 32, 72, 768, 4096, 32768, (8 << 20) / (int)item - piece}) {
            now_rows = rows;
            now_E = E;
            now_in = d_in;
            now_out = d_out;
            const unsigned long long wide = d_in > d_out ? d_in : d_out;
            if ((unsigned long long)rows * (wide / piece) > 0xffffff00ull) continue;
            if ((unsigned long long)d_in * d_out * item >= 1ull << 31) continue;
            now_call = "forward";
            expect_ok(lshmoe_expert_forward(p, p, p, pi, rows, d_in, d_out, E, dtype, LSHMOE_ACT_GELU, p, p, nullptr));
            now_call = "input gradient";
            expect_ok(lshmoe_expert_backward_input(p, p, pi, rows, d_in, d_out, E, dtype, LSHMOE_ACT_RELU, p, p, nullptr));
            now_call = "weight gradient";
            size_t bytes = 0;
            expect_ok(lshmoe_expert_workspace_bytes(rows, d_in, d_out, E, dtype, &bytes));
            // room for two rounds of tiles of 256 KB and the sums, a few more where tiles are many
            if (bytes > (size_t)1 << 30) fail("a workspace of more than 1 GiB");
            expect_ok(lshmoe_expert_backward_weight(p, p, pi, rows, d_in, d_out, E, dtype, p, p, p, bytes, nullptr));
            if (bytes > 0 && lshmoe_expert_backward_weight(p, p, pi, rows, d_in, d_out, E, dtype, p, p, p, bytes - 1, nullptr) !=
                                 LSHMOE_ERR_WORKSPACE)
              fail("a workspace one byte short was taken");
            if (d_in % 32 != 0) continue;
            now_call = "4 bits";
            expect_ok(lshmoe_mx4_quantize(p, rows, d_in, dtype, pb, pb, nullptr));
            expect_ok(lshmoe_mx4_dequantize(pb, pb, rows, d_in, dtype, p, nullptr));
            expect_ok(lshmoe_expert_forward_mx4(pb, pb, pb, pb, p, pi, rows, d_in, d_out, E, dtype, LSHMOE_ACT_NONE, p, nullptr));
          }
  }
  printf("%d launches, %d failures\n", launches, failures);
  return failures || launches < 1000 ? 1 : 0;
}
