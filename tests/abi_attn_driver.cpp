// Host-side paths of the rotary, cache and attention calls, for a build with
// AddressSanitizer and UndefinedBehaviorSanitizer on the host code
// (tests/test_abi_attention_sanitizers.py).  Every call returns before anything is
// enqueued: argument and shape errors over extreme values, workspace queries.
#include <climits>
#include <cmath>
#include <cstdio>

#include "moe.h"

namespace {

int g_calls = 0, g_failures = 0;

void refused(moe_status_t got, int line) {
  ++g_calls;
  if (got == MOE_OK) {
    ++g_failures;
    std::printf("line %d: MOE_OK on invalid arguments\n", line);
  }
}
#define REFUSED(call) refused((call), __LINE__)

template <typename T>
T* at(uintptr_t x) {
  return reinterpret_cast<T*>(x);
}

const int32_t kInts[] = {INT32_MIN, -1, 0, 1, 2, 63, 64, 65, 4096, 65535, 65536, 1 << 20, (1 << 30) + 1, INT32_MAX};
const int64_t kStrides[] = {INT64_MIN, -1024, 0, 8, 1000, 1 << 23, INT64_MAX};
const moe_attn_dims_t kDims[] = {{8, 2, 128}, {1024, 1, 64},  {1024, 1024, 128}, {1, 1, 64},      {0, 0, 0},
                                 {5, 2, 64},  {8, 2, 96},     {-8, -2, 128},     {INT32_MAX, 1, 64}, {INT32_MIN, -1, 64}};

}  // namespace

int main() {
  const uint16_t* x = at<const uint16_t>(0x10000);
  const int32_t* ids = at<const int32_t>(0x20000);
  const float* f = at<const float>(0x30000);
  uint16_t* out = at<uint16_t>(0x40000);
  const moe_kv_cache_t good{at<uint8_t>(0x50000), at<uint8_t>(0x60000), at<float>(0x70000), at<float>(0x80000), 4, 64};

  size_t sum = 0;
  for (const auto& d : kDims)
    for (int32_t a : kInts)
      for (int32_t b : kInts)
        for (int32_t c : kInts) {
          sum += moe_attn_prefill_workspace(d, a, b, c);
          sum += moe_attn_decode_workspace(d, a, b, c);
          g_calls += 2;
        }
  std::printf("workspace queries done (%d)\n", (int)(sum % 2));

  for (const auto& d : kDims) {
    for (int64_t s : kStrides) {
      REFUSED(moe_rope(d, 4, x, s, x, s, ids, f, 10, 128, MOE_ROPE_HALF, out, out, nullptr, nullptr));
      REFUSED(moe_rope_cache(d, 4, x, s, x, s, x, s, ids, f, 10, 128, MOE_ROPE_HALF, ids, good, out, out, nullptr, nullptr));
      REFUSED(moe_attn_prefill(d, 2, 9, 9, 9, x, s, x, s, x, s, ids, ids, 0.1f, 1, out, nullptr, nullptr, 0, nullptr));
      REFUSED(moe_attn_decode(d, 2, x, s, good, ids, 3, ids, 9, nullptr, 0, 0.1f, out, nullptr, nullptr, 0, nullptr));
    }
    // every one of these lacks a pointer, too
    for (int32_t a : kInts) {
      if (a == 0) continue;
      REFUSED(moe_rope(d, a, x, 1 << 20, nullptr, 0, nullptr, f, a, a, MOE_ROPE_HALF, out, nullptr, nullptr, nullptr));
      REFUSED(moe_cache_read(d, good, nullptr, a, a, ids, a, out, out, nullptr, nullptr));
      moe_kv_cache_t c = good;
      c.n_pages = a;
      c.page_size = a;
      REFUSED(moe_cache_read(d, c, nullptr, 2, 3, ids, 4, out, out, nullptr, nullptr));
      REFUSED(moe_attn_decode(d, a, x, 1 << 20, good, nullptr, a, ids, a, ids, a, 0.1f, out, nullptr, nullptr, 0, nullptr));
      REFUSED(moe_attn_prefill(d, a, a, a, a, x, 1 << 20, x, 1 << 20, x, 1 << 20, nullptr, ids, 0.1f, 1, out, nullptr, nullptr,
                               0, nullptr));
      // all pointers, but no workspace, or too many keys
      REFUSED(moe_attn_decode(kDims[0], 65535, x, 1024, good, ids, INT32_MAX, ids, 1 << 20, ids, 1 << 20, 0.1f, out, nullptr,
                              nullptr, 0, nullptr));
    }
    for (float s : {0.0f, -1.0f, NAN, INFINITY, 3.4e38f})
      REFUSED(moe_attn_prefill(d, 2, 9, 9, 9, x, 1024, x, 256, x, 256, ids, ids, s, 1, out, nullptr, nullptr, 0, nullptr));
  }
  for (int32_t rot : kInts)
    for (double v : {0.0, -1.0, (double)NAN, (double)INFINITY, 1e-300})
      for (int scaling : {-1, 1, 2, 7})
        REFUSED(moe_rope_table(moe_rope_cfg_t{rot, scaling, v, v, v, v, v, v}, 10, nullptr, nullptr));

  std::printf("%d checked calls, %d failures\n", g_calls, g_failures);
  return g_failures != 0;
}
