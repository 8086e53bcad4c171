// Host-side paths of the norm and of the calls with 4-bit weights, for a build with
// AddressSanitizer and UndefinedBehaviorSanitizer on the host code
// (tests/test_abi_w4_sanitizers.py).  Every call returns before anything is
// enqueued: argument and shape errors over extreme values, workspace queries.
#include <climits>
#include <cmath>
#include <cstdio>

#include "moe.h"

namespace {

int g_calls = 0, g_failures = 0;

void refused(moe_status_t got, int line) {
  ++g_calls;
  if (got == MOE_OK || got == MOE_ERR_HIP) {
    ++g_failures;
    std::printf("line %d: status %d on invalid arguments\n", line, (int)got);
  }
}
#define REFUSED(call) refused((call), __LINE__)

template <typename T>
T* at(uintptr_t x) {
  return reinterpret_cast<T*>(x);
}

const int32_t kInts[] = {INT32_MIN, -128, -1, 0, 1, 16, 17, 127, 128, 512, 513, 4096, 65536, 75776, 1 << 20, (1 << 30) + 1, INT32_MAX - 127,
                         INT32_MAX - 15, INT32_MAX};
const int64_t kStrides[] = {INT64_MIN, -1024, 0, 8, 1000, 1 << 23, INT64_MAX};

}  // namespace

int main() {
  const uint16_t* x = at<const uint16_t>(0x10000);
  const uint8_t* w = at<const uint8_t>(0x20000);
  const int32_t* ids = at<const int32_t>(0x30000);
  const float* f = at<const float>(0x40000);
  uint16_t* out = at<uint16_t>(0x50000);
  uint8_t* bytes = at<uint8_t>(0x60000);
  float* y = at<float>(0x70000);
  void* odd = at<void>(0x80080);  // a workspace that no call takes

  size_t sum = 0;
  for (int32_t a : kInts)
    for (int32_t b : kInts)
      for (int32_t c : kInts) {
        sum += moe_w4_scale_bytes(a, b, c) + moe_linear_w4_workspace(a, b, c);
        for (int32_t k : {1, 8}) {
          const moe_dims_t d{a, b, 8, k};
          sum += moe_expert_ffn_w4_workspace(d, c) + moe_ffn_layer_w4_workspace(d, c);
        }
        g_calls += 6;
        // Good arguments as far as the workspace, which is misaligned; too large grids are refused behind it.
        if (a > 0) REFUSED(moe_linear_w4(x, 1 << 30, a, b, w, w, c, nullptr, out, INT64_MAX & ~(int64_t)7, MOE_BF16, odd, SIZE_MAX, nullptr));
      }
  std::printf("workspace queries done (%d)\n", (int)(sum % 2));
  REFUSED(moe_linear_w4(x, 128, 100000, 128, w, w, INT32_MAX - 15, nullptr, out, (int64_t)1 << 31, MOE_F32, bytes, SIZE_MAX, nullptr));

  for (int32_t a : kInts)
    for (int32_t b : kInts) {
      // codes without scales
      const moe_norm_cfg_t cfg{1e-6f, 0.0f, b, MOE_BF16, MOE_F32};
      if (a != 0)
        for (int64_t s : kStrides)
          REFUSED(moe_add_norm(x, s, x, s, nullptr, a, 256, cfg, nullptr, 0, out, s, bytes, nullptr, nullptr));
      REFUSED(moe_add_norm(nullptr, 256, nullptr, 0, nullptr, 1, a, cfg, nullptr, 0, out, 256, nullptr, nullptr, nullptr));
      for (int32_t c : kInts) {
        if (a != 0) {
          REFUSED(moe_quant_weight_w4(nullptr, a, b, c, bytes, bytes, nullptr));
          REFUSED(moe_pack_weight_w4(w, w, a, b, c, nullptr, bytes, nullptr, nullptr));
        }
        if (a == 0) continue;
        for (int32_t e : {-1, 0, 1, 1024, 1025, INT32_MAX}) {
          const moe_dims_t d{b, c, e, 1};
          REFUSED(moe_expert_ffn_w4(d, a, x, ids, ids, w, w, w, w, w, w, y, odd, SIZE_MAX, nullptr));
          REFUSED(moe_ffn_layer_w4(d, a, x, ids, f, w, w, w, w, w, w, out, nullptr, odd, SIZE_MAX, nullptr));
          REFUSED(moe_expert_ffn_w4(d, a, x, ids, ids, w, w, w, w, w, nullptr, y, bytes, SIZE_MAX, nullptr));
        }
      }
    }
  for (float eps : {0.0f, -1.0f, NAN, INFINITY, 1e-13f, 1e-45f})
    REFUSED(moe_add_norm(x, 256, nullptr, 0, nullptr, 1, 256, moe_norm_cfg_t{eps, 0.0f, 1, MOE_BF16, MOE_BF16}, nullptr, 0, out, 256,
                         nullptr, nullptr, nullptr));
  for (float offset : {NAN, INFINITY, -INFINITY})
    REFUSED(moe_add_norm(x, 256, nullptr, 0, nullptr, 1, 256, moe_norm_cfg_t{1e-6f, offset, 1, MOE_BF16, MOE_BF16}, nullptr, 0, out,
                         256, nullptr, nullptr, nullptr));
  std::printf("%d calls, %d failures\n", g_calls, g_failures);
  return g_failures != 0;
}
