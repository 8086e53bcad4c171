// Attention of one token per sequence over the paged e4m3 cache.
//
// The G query heads of a key/value head are the columns of 16x16x32 bf16
// MFMAs (16 of them, padded), so a key's codes are read and converted once for
// the group:
//   S^T = K Q^T   keys' codes go from the pages to registers as the first
//                 operand (lane: key lane % 16, 16 codes at 16 (lane / 16) of
//                 each 64), converted to bf16 exactly; a lane ends with the scores
//                 of query lane % 16 for keys 4 (lane / 16) + i
//   O^T = V^T P^T values' codes go through LDS and come back transposed
//                 (ds_read_b64_tr_b8) in the order of keys that the scores have
// Scales stay fp32: a key's multiplies its score, a value's its softmax numerator,
// which is rounded to bf16 once.
#include <math.h>

#include <algorithm>

#include "attention.h"

namespace moe {

namespace {

struct DecodeArgs {
  const uint16_t* q;
  int64_t q_stride;
  moe_kv_cache_t cache;
  const int32_t *pages, *lens, *prefix_pages;
  uint16_t* out;
  int32_t* status;
  int B, width, prefix_len, kv_heads, group, page_shift;
  float c;  // scale * log2(e)
};

constexpr int kKeys = 32;   // keys per step of a wave
constexpr int kWaves = 4;
constexpr int kCols = 16;   // queries per product

// One wave's running softmax: lane's query is column lane % 16.
template <int D>
struct Running {
  v4f o[D / 16];  // O^T: rows 16 i + 4 (lane / 16) + 0..3
  float m, l;     // l: this lane's keys only, summed over the lane groups at the end
};

__device__ __forceinline__ int page_at(const DecodeArgs& a, const int32_t* pages, int index) {
  const int p = pages[index];
  if (p >= 0 && p < a.cache.n_pages) return p;
  if (a.status && (threadIdx.x & 63) == 0) atomicOr(a.status, MOE_DEV_BAD_PAGE);
  return 0;  // in bounds; the outputs that need it are unspecified
}

// Keys [t0, t0 + 32) of the `len` that `pages` hold.
template <int D>
__device__ __forceinline__ void step(const DecodeArgs& a, const int32_t* pages, int len, int t0, int kvh,
                                     const v8bf (&qf)[D / 32], uint8_t* lds_v, Running<D>& run) {
  const int lane = threadIdx.x & 63, g = lane >> 4, c16 = lane & 15;
  const int mask = a.cache.page_size - 1, last = len - 1;
  // each half of 16 keys lies in one page; keys behind the end repeat the last
  int64_t base[2];
  int row0[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int t = min(t0 + 16 * u, last) & ~15;
    base[u] = ((int64_t)page_at(a, pages, t >> a.page_shift) * a.kv_heads + kvh) << a.page_shift;
    row0[u] = t;
  }
  v4f s[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int t = min(row0[u] + c16, last) & mask;
    const uint8_t* krow = a.cache.k + (base[u] + t) * D + 16 * g;
    s[u] = v4f{};
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      const uint4 x = *reinterpret_cast<const uint4*>(krow + 64 * i);
      s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(e4m3x8_to_bf16(x.x, x.y), qf[2 * i], s[u], 0, 0, 0);
      s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(e4m3x8_to_bf16(x.z, x.w), qf[2 * i + 1], s[u], 0, 0, 0);
    }
  }
  // values to LDS: rows of D codes, 16-byte chunks swizzled
  constexpr int kChunks = D / 16;
  const auto place = [](int row, int c) {
    const int f = D == 128 ? ((row >> 1) & 3) | ((row >> 2) & 4) : ((row >> 2) & 1) | ((row >> 3) & 2);
    return row * D + ((c ^ f) * 16);
  };
#pragma unroll
  for (int i = 0; i < 32 * kChunks / 64; ++i) {
    const int p = 64 * i + lane, row = p / kChunks, c = p % kChunks, u = row >> 4;
    const int t = min(row0[u] + (row & 15), last) & mask;
    *reinterpret_cast<uint4*>(lds_v + place(row, c)) =
        *reinterpret_cast<const uint4*>(a.cache.v + ((u ? base[1] : base[0]) + t) * D + 16 * c);
  }
  float vs[2][4];
  float top = -INFINITY;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int64_t at = base[u] + (row0[u] & mask) + 4 * g;
    const float4 ks = *reinterpret_cast<const float4*>(a.cache.k_scale + at);
    const float4 vv = *reinterpret_cast<const float4*>(a.cache.v_scale + at);
    const float kk[4] = {ks.x, ks.y, ks.z, ks.w}, vx[4] = {vv.x, vv.y, vv.z, vv.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool there = t0 + 16 * u + 4 * g + i < len;  // a slot behind the end may hold any bits
      s[u][i] = there ? s[u][i] * (kk[i] * a.c) : -INFINITY;
      vs[u][i] = there ? vx[i] : 0.0f;
      top = fmaxf(top, s[u][i]);
    }
  }
  top = fmaxf(top, __shfl_xor(top, 16, 64));
  top = fmaxf(top, __shfl_xor(top, 32, 64));
  const float m = fmaxf(run.m, top), alpha = __builtin_amdgcn_exp2f(run.m - m);
  run.m = m;
  float sum = 0.0f;
  union {
    v8bf v;
    uint32_t x[4];
  } p;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    float e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      e[i] = __builtin_amdgcn_exp2f(s[u][i] - m);
      sum += e[i];
      e[i] *= vs[u][i];
    }
    p.x[2 * u] = pack_bf16(e[0], e[1]);
    p.x[2 * u + 1] = pack_bf16(e[2], e[3]);
  }
  run.l = run.l * alpha + sum;
  // lane j of a 16-lane group gives the address of row j / 2, half j % 2 of an 8 x 16 block and gets column j:
  // rows 0..3 are keys 4 g + 0..3, rows 4..7 keys 16 + 4 g + 0..3
  const int j = c16 >> 1, row = (j < 4 ? 0 : 12) + 4 * g + j;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    const v2i x = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
        (__attribute__((address_space(3))) v2i*)(lds_v + place(row, i) + 8 * (c16 & 1)));
    run.o[i] *= alpha;
    run.o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(e4m3x8_to_bf16(x[0], x[1]), p.v, run.o[i], 0, 0, 0);
  }
}

// One workgroup per (sequence, key/value head, block of 16 of its queries); the
// waves take every fourth step and are joined through LDS.
template <int D>
__global__ __launch_bounds__(64 * kWaves) void attn_decode_kernel(DecodeArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t lds_v[kWaves][kKeys * D];
  __shared__ float lds_o[kWaves][kCols][D + 4];
  __shared__ float lds_m[kWaves][kCols], lds_l[kWaves][kCols];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, c16 = lane & 15;
  const int b = blockIdx.x, kvh = blockIdx.y, col0 = blockIdx.z * kCols;
  const int cols = min(kCols, a.group - col0);
  const int head0 = kvh * a.group + col0;

  v8bf qf[D / 32];
  const uint16_t* qrow = a.q + b * a.q_stride + (head0 + min(c16, cols - 1)) * D + 16 * g;
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    qf[2 * i] = *reinterpret_cast<const v8bf*>(qrow + 64 * i);
    qf[2 * i + 1] = *reinterpret_cast<const v8bf*>(qrow + 64 * i + 8);
  }
  Running<D> run;
  run.m = kNoScore;
  run.l = 0.0f;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) run.o[i] = v4f{};

  int len = a.lens[b];
  const int64_t most = min((int64_t)a.width << a.page_shift, (int64_t)0x7fffffff);
  if (len < 0 || len > most) {
    if (a.status && threadIdx.x == 0) atomicOr(a.status, MOE_DEV_BAD_LENGTH);
    len = len < 0 ? 0 : (int)most;
  }
  for (int t = wave * kKeys; t < a.prefix_len; t += kWaves * kKeys)
    step<D>(a, a.prefix_pages, a.prefix_len, t, kvh, qf, lds_v[wave], run);
  for (int t = wave * kKeys; t < len; t += kWaves * kKeys)
    step<D>(a, a.pages + (int64_t)b * a.width, len, t, kvh, qf, lds_v[wave], run);

  run.l += __shfl_xor(run.l, 16, 64);
  run.l += __shfl_xor(run.l, 32, 64);
  if (g == 0) {
    lds_m[wave][c16] = run.m;
    lds_l[wave][c16] = run.l;
  }
#pragma unroll
  for (int i = 0; i < D / 16; ++i) *reinterpret_cast<v4f*>(&lds_o[wave][c16][16 * i + 4 * g]) = run.o[i];
  __syncthreads();
  for (int p = threadIdx.x; p < cols * D / 4; p += 64 * kWaves) {
    const int col = p / (D / 4), d = p % (D / 4) * 4;
    float m = kNoScore;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) m = fmaxf(m, lds_m[w][col]);
    float l = 0.0f;
    v4f o = {};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(lds_m[w][col] - m);
      l += lds_l[w][col] * f;
      o += *reinterpret_cast<const v4f*>(&lds_o[w][col][d]) * f;
    }
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    *reinterpret_cast<uint2*>(a.out + ((int64_t)b * (a.kv_heads * a.group) + head0 + col) * D + d) =
        make_uint2(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv));
  }
}

template <int D>
moe_status_t launch_decode(const DecodeArgs& a, hipStream_t stream) {
  MOE_LAUNCH("attn_decode", attn_decode_kernel<D>, dim3(a.B, a.kv_heads, (a.group + kCols - 1) / kCols),
             dim3(64 * kWaves), 0, stream, a);
  return check_launch("moe_attn_decode");
}

}  // namespace

}  // namespace moe

using namespace moe;

extern "C" size_t moe_attn_decode_workspace(moe_attn_dims_t d, int32_t B, int32_t max_len, int32_t prefix_len) {
  (void)d;
  (void)B;
  (void)max_len;
  (void)prefix_len;
  return 0;
}

extern "C" moe_status_t moe_attn_decode(moe_attn_dims_t d, int32_t B, const uint16_t* q, int64_t q_stride,
                                        moe_kv_cache_t cache, const int32_t* page_table, int32_t table_width,
                                        const int32_t* lens, int32_t max_len, const int32_t* prefix_pages,
                                        int32_t prefix_len, float scale, uint16_t* out, int32_t* dev_status, void* ws,
                                        size_t ws_bytes, hipStream_t stream) {
  moe_status_t st = check_attn_dims(d, "moe_attn_decode");
  if (st != MOE_OK) return st;
  if ((st = check_cache(cache, "moe_attn_decode")) != MOE_OK) return st;
  if (B < 0 || B > 65535 || table_width < 0 || max_len < 0 || prefix_len < 0)
    return fail(MOE_ERR_INVALID_ARG, "moe_attn_decode: B=%d (at most 65535) table_width=%d max_len=%d prefix_len=%d", B,
                table_width, max_len, prefix_len);
  if (!(scale > 0.0f) || !isfinite(scale * kLog2e)) return fail(MOE_ERR_INVALID_ARG, "moe_attn_decode: scale=%g", scale);
  if (B == 0) return MOE_OK;
  if ((st = check_rows(q, q_stride, d.q_heads, d.head_dim, "moe_attn_decode", "q")) != MOE_OK) return st;
  if (!page_table || !lens || !out || (prefix_len > 0 && !prefix_pages))
    return fail(MOE_ERR_INVALID_ARG, "moe_attn_decode: null pointer");
  if (!aligned(out, 16)) return fail(MOE_ERR_INVALID_ARG, "moe_attn_decode: out must be 16-byte aligned");
  const size_t need = moe_attn_decode_workspace(d, B, max_len, prefix_len);
  if (need && (!ws || ws_bytes < need || !aligned(ws, 256)))
    return fail(MOE_ERR_WORKSPACE, "moe_attn_decode: workspace %zu bytes, needs %zu, 256-byte aligned", ws_bytes, need);
  const DecodeArgs a{q, q_stride, cache, page_table, lens, prefix_pages, out, dev_status, B, table_width, prefix_len,
                     d.kv_heads, d.q_heads / d.kv_heads, __builtin_ctz((unsigned)cache.page_size), scale * kLog2e};
  return d.head_dim == 64 ? launch_decode<64>(a, stream) : launch_decode<128>(a, stream);
}
