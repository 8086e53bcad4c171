// The calls with 4-bit weights: checks, workspaces, and which kernel runs.
#include <algorithm>

#include "w4.h"
#include "w4_rows.h"

namespace moe {

bool w4_few_fits(int32_t K);
int w4_few_parts(int32_t K);
moe_status_t run_w4_few(const W4Args& a, bool gateup, int64_t rows, hipStream_t stream);
moe_status_t run_w4_few_slots(const W4Args& a, int rows, const W4Slots& slots, hipStream_t stream);
bool w4_down_combine_fits(int32_t K, int slots);
moe_status_t run_w4_down_combine(const moe_dims_t& d, int tokens, const uint16_t* h, const W4Slots& s, const uint8_t* w,
                                 const uint8_t* w_s, const float* topk_w, uint16_t* out, hipStream_t stream);
W4Cut w4_gemm_cut(int64_t rows, int32_t K, int32_t N);
moe_status_t run_w4_gemm(const W4Args& a, bool gateup, int64_t rows, hipStream_t stream);

namespace {

constexpr int kFewRows = 16;  // rows of one matrix that w4_few takes

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Experts with a few rows each: w4_few streams their weights faster than the GEMM's smallest tiles (a layer of 7168 x 2048,
// 256 experts of 8 a token: 380 against 428 us at 16 tokens, 832 against 893 at 64, 1010 against 1026 at 256; 2048 x 768,
// 128 experts of 8: 53 against 61 at 16, 78 against 75 at 128; 4096 x 1536, 16 experts of 2: 46 against 49 at 33, 48
// against 49 at 64), and slower where they have more than 8 (the same layers, 12 rows: 89 against 78 and 54 against 49).
bool few_experts(const W4Args& a, int64_t rows) {
  return rows <= kFewMaxRows && rows <= 8 * (int64_t)a.E && w4_few_fits(a.K);
}

moe_status_t run_experts(const W4Args& a, bool gateup, int64_t rows, hipStream_t stream) {
  return few_experts(a, rows) ? run_w4_few(a, gateup, rows, stream) : run_w4_gemm(a, gateup, rows, stream);
}

// One matrix: whether w4_few takes it.
bool few_linear(int32_t T, int32_t K) { return T <= kFewRows && w4_few_parts(K) <= w4_most_parts(kFewRows); }

// Parts of K that one matrix is multiplied in.
int linear_parts(int32_t T, int32_t K, int32_t N) {
  return few_linear(T, K) ? w4_few_parts(K) : w4_gemm_cut(T, K, N).parts;
}

// Bytes of the sums of `rows` = parts * T rows.
size_t sums_bytes(int64_t rows, int32_t N) { return align256((size_t)rows * N * sizeof(float)); }

// out = the parts' sums in their order (+ bias), four neighbouring outputs a lane.
__global__ __launch_bounds__(256) void w4_join_kernel(W4Args p) {
  const int n = (int)(blockIdx.x * blockDim.x + threadIdx.x) * 4;
  if (n >= p.N) return;
  const int64_t step = p.x_rows * p.N;
  for (int64_t row = blockIdx.y; row < p.x_rows; row += gridDim.y) {
    const float* from = p.partial + row * p.N + n;
    v4f v = *reinterpret_cast<const v4f*>(from);
#pragma unroll 4
    for (int s = 1; s < p.splits; ++s) v += *reinterpret_cast<const v4f*>(from + s * step);
    w4_store(p, row, n, v);
  }
}

moe_status_t run_linear(const W4Args& a, int32_t T, hipStream_t stream) {
  const moe_status_t st = few_linear(T, a.K) ? run_w4_few(a, false, T, stream) : run_w4_gemm(a, false, T, stream);
  if (st != MOE_OK || a.splits <= 1) return st;
  MOE_LAUNCH("w4_join", w4_join_kernel, dim3((unsigned)(((int64_t)a.N / 4 + 255) / 256), (unsigned)std::min(T, 1024)), dim3(256), 0,
             stream, a);
  return check_launch("w4_join");
}

moe_status_t check_w4_dims(const moe_dims_t& d, int32_t T, const char* who) {
  if (d.hidden <= 0 || d.inter <= 0 || d.n_experts < 1 || d.n_experts > 1024 || d.topk < 1 || d.topk > 32 ||
      d.topk > d.n_experts || T < 0)
    return fail(MOE_ERR_INVALID_ARG, "%s: dims H=%d I=%d E=%d k=%d, T=%d", who, d.hidden, d.inter, d.n_experts, d.topk, T);
  if (d.hidden % kBlock || d.inter % kBlock)
    return fail(MOE_ERR_UNSUPPORTED_SHAPE, "%s: H=%d, I=%d must be multiples of 128", who, d.hidden, d.inter);
  if ((int64_t)T * d.topk > 0x7fffffff) return fail(MOE_ERR_UNSUPPORTED_SHAPE, "%s: T*k overflows", who);
  return MOE_OK;
}

moe_status_t check_w4_stacks(const void* x, const uint8_t* const (&w)[6], const void* out, const char* who) {
  for (const uint8_t* m : w)
    if (!m) return fail(MOE_ERR_INVALID_ARG, "%s: null pointer", who);
  if (!x || !out) return fail(MOE_ERR_INVALID_ARG, "%s: null pointer", who);
  for (const uint8_t* m : w)
    if (!aligned(m, 16)) return fail(MOE_ERR_INVALID_ARG, "%s: misaligned weights (16 bytes needed)", who);
  if (!aligned(x, 16) || !aligned(out, 16)) return fail(MOE_ERR_INVALID_ARG, "%s: misaligned pointer (16 bytes needed)", who);
  return MOE_OK;
}

moe_status_t check_workspace(const void* ws, size_t have, size_t need, const char* who) {
  if (need && (!ws || have < need)) return fail(MOE_ERR_WORKSPACE, "%s: workspace %zu bytes < %zu", who, have, need);
  if (!aligned(ws, 256)) return fail(MOE_ERR_INVALID_ARG, "%s: workspace must be 256-byte aligned", who);
  return MOE_OK;
}

// h is bf16: the matrix instruction of the down projection takes 16 bits, and h in two such parts would double its
// products.  (2.3e-3 of the output's norm against 1.7e-3 for the output's own rounding.)  All sums are fp32.
W4Args gateup_args(const moe_dims_t& d, int32_t T, const uint16_t* x, const uint8_t* const (&w)[6], uint16_t* h) {
  W4Args g{};
  g.x = x; g.x_stride = d.hidden; g.x_rows = T; g.topk = d.topk; g.E = d.n_experts;
  g.w0 = w[0]; g.s0 = w[1]; g.w1 = w[2]; g.s1 = w[3];
  g.N = d.inter; g.K = d.hidden; g.out16 = h; g.out_stride = d.inter;
  return g;
}

moe_status_t expert_ffn_w4(const moe_dims_t& d, int32_t T, const uint16_t* x, const int32_t* offsets, const int32_t* src,
                           const uint8_t* const (&w)[6], uint16_t* h, float* y, hipStream_t stream) {
  const int64_t rows = (int64_t)T * d.topk;
  W4Args g = gateup_args(d, T, x, w, h);
  g.sorted_src = src; g.offsets = offsets;
  const moe_status_t st = run_experts(g, true, rows, stream);
  if (st != MOE_OK) return st;
  W4Args dn{};
  dn.x = h; dn.x_stride = d.inter; dn.x_rows = rows;
  dn.offsets = offsets; dn.E = d.n_experts;
  dn.w0 = w[4]; dn.s0 = w[5];
  dn.N = d.hidden; dn.K = d.inter; dn.out32 = y; dn.out_stride = d.hidden;
  return run_experts(dn, false, rows, stream);
}

struct W4LayerLayout {
  size_t offsets, src, dest, list, y, perm, h, total;
};

W4LayerLayout w4_layer_layout(const moe_dims_t& d, int32_t T) {
  W4LayerLayout L{};
  const size_t R = (size_t)T * d.topk;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += align256(bytes);
    return here;
  };
  L.offsets = take((size_t)(d.n_experts + 1) * sizeof(int32_t));
  L.src = take(R * sizeof(int32_t));
  L.dest = take(R * sizeof(int32_t));
  L.list = take((kSortSlots + 1) * sizeof(int2));
  L.y = take(R * d.hidden * sizeof(float));
  L.perm = take(moe_permute_workspace(T, d.topk, d.n_experts));
  L.h = take(moe_expert_ffn_w4_workspace(d, T));
  L.total = at;
  return L;
}

}  // namespace

}  // namespace moe

using namespace moe;

extern "C" size_t moe_linear_w4_workspace(int32_t T, int32_t K, int32_t N) {
  if (T <= 0 || K <= 0 || N <= 0 || K % kBlock || N % 16) return 0;
  // Sums of the parts of K, of this T and every smaller one.  Of 16 j + 1 to 16 j + 16 rows the first has the most parts:
  // within them a cut's estimate grows by its sums alone, and by more the more parts it has.
  int64_t most = 0;
  int32_t first = 1;
  if (few_linear(1, K)) {
    if (w4_few_parts(K) > 1) most = (int64_t)w4_few_parts(K) * std::min(T, kFewRows);
    first = kFewRows + 1;
  }
  for (; first <= T && w4_most_parts(first) > 1; first += 16) {
    const int parts = w4_gemm_cut(first, K, N).parts;
    if (parts > 1) most = std::max(most, (int64_t)parts * std::min(T, first + 15));
  }
  return sums_bytes(most, N);
}

extern "C" moe_status_t moe_linear_w4(const uint16_t* x, int64_t x_stride, int32_t T, int32_t K, const uint8_t* w,
                                      const uint8_t* w_s, int32_t N, const uint16_t* bias, void* out, int64_t out_stride,
                                      moe_float_t out_type, void* ws, size_t ws_bytes, hipStream_t stream) {
  if (T < 0 || K <= 0 || N <= 0) return fail(MOE_ERR_INVALID_ARG, "moe_linear_w4: T=%d K=%d N=%d", T, K, N);
  if (out_type != MOE_BF16 && out_type != MOE_F32) return fail(MOE_ERR_INVALID_ARG, "moe_linear_w4: out_type=%d", (int)out_type);
  if (K % kBlock || N % 16)
    return fail(MOE_ERR_UNSUPPORTED_SHAPE, "moe_linear_w4: K=%d (a multiple of 128), N=%d (of 16)", K, N);
  if (T == 0) return MOE_OK;
  if (!x || !w || !w_s || !out) return fail(MOE_ERR_INVALID_ARG, "moe_linear_w4: null pointer");
  if (!aligned(x, 16) || !aligned(w, 16) || !aligned(w_s, 16) || !aligned(out, 16) || !aligned(bias, 8))
    return fail(MOE_ERR_INVALID_ARG, "moe_linear_w4: misaligned pointer");
  if (x_stride < K || x_stride % 8 || out_stride < N || out_stride % 8)
    return fail(MOE_ERR_INVALID_ARG, "moe_linear_w4: strides %lld of x, %lld of out must be multiples of 8, at least %d and %d",
                (long long)x_stride, (long long)out_stride, K, N);
  const int parts = linear_parts(T, K, N);
  const moe_status_t st = check_workspace(ws, ws_bytes, parts > 1 ? sums_bytes((int64_t)parts * T, N) : 0, "moe_linear_w4");
  if (st != MOE_OK) return st;
  W4Args a{};
  a.x = x; a.x_stride = x_stride; a.x_rows = T;
  a.w0 = w; a.s0 = w_s; a.bias = bias; a.N = N; a.K = K;
  a.out32 = out_type == MOE_F32 ? static_cast<float*>(out) : nullptr;
  a.out16 = out_type == MOE_F32 ? nullptr : static_cast<uint16_t*>(out);
  a.out_stride = out_stride;
  a.splits = parts;
  a.partial = static_cast<float*>(ws);
  return run_linear(a, T, stream);
}

extern "C" size_t moe_expert_ffn_w4_workspace(moe_dims_t d, int32_t T) {
  if (T < 0 || d.inter <= 0 || d.topk <= 0) return 0;
  return align256((size_t)T * d.topk * d.inter * sizeof(uint16_t));
}

extern "C" moe_status_t moe_expert_ffn_w4(moe_dims_t d, int32_t T, const uint16_t* x, const int32_t* expert_offsets,
                                          const int32_t* sorted_src, const uint8_t* w_gate, const uint8_t* s_gate,
                                          const uint8_t* w_up, const uint8_t* s_up, const uint8_t* w_down,
                                          const uint8_t* s_down, float* y_rows, void* ws, size_t ws_bytes,
                                          hipStream_t stream) {
  moe_status_t st = check_w4_dims(d, T, "moe_expert_ffn_w4");
  if (st != MOE_OK) return st;
  if (T == 0) return MOE_OK;
  const uint8_t* const w[6] = {w_gate, s_gate, w_up, s_up, w_down, s_down};
  st = check_w4_stacks(x, w, y_rows, "moe_expert_ffn_w4");
  if (st != MOE_OK) return st;
  if (!expert_offsets || !sorted_src) return fail(MOE_ERR_INVALID_ARG, "moe_expert_ffn_w4: null pointer");
  st = check_workspace(ws, ws_bytes, moe_expert_ffn_w4_workspace(d, T), "moe_expert_ffn_w4");
  if (st != MOE_OK) return st;
  return expert_ffn_w4(d, T, x, expert_offsets, sorted_src, w, static_cast<uint16_t*>(ws), y_rows, stream);
}

extern "C" size_t moe_ffn_layer_w4_workspace(moe_dims_t d, int32_t T) {
  if (check_w4_dims(d, T, "moe_ffn_layer_w4_workspace") != MOE_OK) return 0;
  return w4_layer_layout(d, T).total;
}

extern "C" moe_status_t moe_ffn_layer_w4(moe_dims_t d, int32_t T, const uint16_t* x, const int32_t* topk_ids,
                                         const float* topk_w, const uint8_t* w_gate, const uint8_t* s_gate,
                                         const uint8_t* w_up, const uint8_t* s_up, const uint8_t* w_down,
                                         const uint8_t* s_down, uint16_t* out, int32_t* dev_status, void* ws,
                                         size_t ws_bytes, hipStream_t stream) {
  moe_status_t st = check_w4_dims(d, T, "moe_ffn_layer_w4");
  if (st != MOE_OK) return st;
  if (T == 0) return MOE_OK;
  const uint8_t* const w[6] = {w_gate, s_gate, w_up, s_up, w_down, s_down};
  st = check_w4_stacks(x, w, out, "moe_ffn_layer_w4");
  if (st != MOE_OK) return st;
  if (!topk_ids || !topk_w) return fail(MOE_ERR_INVALID_ARG, "moe_ffn_layer_w4: null pointer");
  const W4LayerLayout L = w4_layer_layout(d, T);
  st = check_workspace(ws, ws_bytes, L.total, "moe_ffn_layer_w4");
  if (st != MOE_OK) return st;
  uint8_t* b = static_cast<uint8_t*>(ws);
  int32_t* offsets = reinterpret_cast<int32_t*>(b + L.offsets);
  int32_t* src = reinterpret_cast<int32_t*>(b + L.src);
  int32_t* dest = reinterpret_cast<int32_t*>(b + L.dest);
  float* y = reinterpret_cast<float*>(b + L.y);
  uint16_t* h = reinterpret_cast<uint16_t*>(b + L.h);
  const int64_t slots = (int64_t)T * d.topk;
  if (w4_few_fits(d.hidden) && slots <= kSortSlots && w4_down_combine_fits(d.inter, (int)slots)) {
    // A few slots: two launches.  Gate/up sorts them itself, the down projection and the combine follow together.
    const W4Slots s{topk_ids, dev_status, reinterpret_cast<int2*>(b + L.list), dest};
    st = run_w4_few_slots(gateup_args(d, T, x, w, h), (int)slots, s, stream);
    if (st != MOE_OK) return st;
    return run_w4_down_combine(d, T, h, s, w_down, s_down, topk_w, out, stream);
  }
  st = moe_permute(topk_ids, T, d.topk, d.n_experts, offsets, src, dest, dev_status, b + L.perm, L.h - L.perm, stream);
  if (st != MOE_OK) return st;
  st = expert_ffn_w4(d, T, x, offsets, src, w, h, y, stream);
  if (st != MOE_OK) return st;
  return moe_combine(y, dest, topk_w, T, d.topk, d.hidden, out, stream);
}
