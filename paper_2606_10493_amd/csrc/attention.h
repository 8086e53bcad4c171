// What the rotary, cache and attention kernels share.
#pragma once

#include "common.h"

namespace moe {

typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef int v2i __attribute__((ext_vector_type(2)));

// The running maximum of scores before the first key: the lowest finite value, so
// that no score lies below it but -inf, a masked key's, and exp2(-inf - m) is 0
// against it, never exp2(-inf + inf).
constexpr float kNoScore = -3.402823466e+38f;
constexpr float kLog2e = 1.44269504088896341f;

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const v2f f = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, v2bf));
}

// Eight e4m3 codes -> eight bf16 (exact: e4m3 has 3 bits of mantissa).
__device__ __forceinline__ v8bf e4m3x8_to_bf16(uint32_t lo, uint32_t hi) {
  union {
    v8bf v;
    v2bf p[4];
  } r;
  r.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
  r.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
  r.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
  r.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
  return r.v;
}

// Inclusive sum over the wave's lanes up to this one (register moves between
// neighbouring lanes, rows of 16 and halves).
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);   // row_shr:1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);   // row_shr:2
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);   // row_shr:4
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);   // row_shr:8
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast:15 into rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast:31 into rows 2 and 3
  return x;
}

// Host side: the checks every attention-side call makes of its dims, a row
// stride of `heads` heads and a cache.
inline moe_status_t check_attn_dims(const moe_attn_dims_t& d, const char* who) {
  if (d.q_heads < 1 || d.kv_heads < 1 || d.head_dim < 1)
    return fail(MOE_ERR_INVALID_ARG, "%s: q_heads=%d kv_heads=%d head_dim=%d", who, d.q_heads, d.kv_heads, d.head_dim);
  if (d.q_heads > 1024 || d.q_heads % d.kv_heads || (d.head_dim != 64 && d.head_dim != 128))
    return fail(MOE_ERR_UNSUPPORTED_SHAPE, "%s: q_heads=%d (at most 1024, a multiple of kv_heads=%d), head_dim=%d (64 or 128)",
                who, d.q_heads, d.kv_heads, d.head_dim);
  return MOE_OK;
}

constexpr int64_t kMaxStride = (int64_t)1 << 23;
inline moe_status_t check_rows(const void* p, int64_t stride, int32_t heads, int32_t dim, const char* who,
                               const char* name) {
  if (!p) return fail(MOE_ERR_INVALID_ARG, "%s: %s is NULL", who, name);
  if (!aligned(p, 16)) return fail(MOE_ERR_INVALID_ARG, "%s: %s must be 16-byte aligned", who, name);
  if (stride < (int64_t)heads * dim || stride % 8 || stride >= kMaxStride)
    return fail(MOE_ERR_INVALID_ARG, "%s: stride %lld of %s must be a multiple of 8, from %lld to below 2^23", who, (long long)stride,
                name, (long long)heads * dim);
  return MOE_OK;
}

inline moe_status_t check_cache(const moe_kv_cache_t& c, const char* who) {
  if (c.n_pages < 1 || c.page_size < 16 || c.page_size > 1024 || (c.page_size & (c.page_size - 1)))
    return fail(MOE_ERR_INVALID_ARG, "%s: n_pages=%d, page_size=%d (a power of two, 16..1024)", who, c.n_pages, c.page_size);
  if (!c.k || !c.v || !c.k_scale || !c.v_scale) return fail(MOE_ERR_INVALID_ARG, "%s: NULL in the cache", who);
  if (!aligned(c.k, 16) || !aligned(c.v, 16) || !aligned(c.k_scale, 16) || !aligned(c.v_scale, 16))
    return fail(MOE_ERR_INVALID_ARG, "%s: the cache's arrays must be 16-byte aligned", who);
  return MOE_OK;
}

}  // namespace moe
