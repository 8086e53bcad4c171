// What the kernels with 4-bit weights share: the packed layout (moe_pack_weight_w4)
// and the expansion of its codes.
#pragma once

#include "common.h"

namespace moe {

typedef __bf16 w4_bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 w4_bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kW4Group = MOE_W4_GROUP;
constexpr int kW4TileBytes = 16 * kBlock / 2;          // 16 rows x 128 columns of codes
constexpr int kW4ScaleCols = 512;                      // columns whose scales lie together
constexpr int kW4ScaleTile = 16 * kW4ScaleCols / kW4Group;  // bytes of 16 rows' scales of them
constexpr int kW4MaxScale = 252;
constexpr int kW4NoScale = 255;

// Eight e2m1 codes (a dword, the first column lowest) times 2^(byte - 127) -> eight
// bf16.  Exact: one bit of mantissa.  The instruction takes the exponent field of
// `scale` and nothing else of it (every byte, with 16384 signs and mantissas each: the same bits).
__device__ __forceinline__ w4_bf16x8 w4_expand(uint32_t codes, float scale) {
  const w4_bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
  const w4_bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
  const w4_bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
  const w4_bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
  return w4_bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Byte j of a row's four scales of a 128-column block in the exponent field, as w4_expand takes it; other bytes around it.
__device__ __forceinline__ float w4_scale(uint32_t four, int j) {
  return __uint_as_float(j == 3 ? four >> 1 : four << (23 - 8 * j));
}

inline int64_t w4_scale_chunks(int32_t cols) { return ((int64_t)cols + kW4ScaleCols - 1) / kW4ScaleCols; }

// A launch has less than 2^32 threads.
inline int64_t w4_max_blocks(int threads) { return ((int64_t)1 << 32) / threads - 1; }

// Rows of activations times packed matrices: out[row, n] = sum_k x[src(row), k] W[n, k].
struct W4Args {
  const uint16_t* x;          // bf16 rows
  int64_t x_stride;
  int64_t x_rows;
  const int32_t* sorted_src;  // row p reads x row sorted_src[p] / topk; NULL: x row p
  int topk;
  const int32_t* offsets;     // [E + 1] rows of each expert; NULL: one matrix for rows 0 .. x_rows - 1
  int E;
  const uint8_t *w0, *s0;     // packed codes and scales [E, N, K]
  const uint8_t *w1, *s1;     // the up projection's
  const uint16_t* bias;       // [N] or NULL
  int N, K;
  float* out32;               // one of the two
  uint16_t* out16;
  int64_t out_stride;
  int splits;                 // parts of K, each a workgroup's, that write their sums to partial [splits, x_rows, N]; 0, 1: none
  float* partial;
};

// A few slots' experts, sorted by the gate/up launch for the launches behind it (device memory).
struct W4Slots {
  const int32_t* ids;   // [slots], the router's
  int32_t* dev_status;  // or NULL
  int2* list;           // [kSortSlots + 1] row tiles, the last entry their number
  int32_t* dest_row;    // [slots]
};

// This workgroup's part of K, in blocks (a whole number of `unit`); a part of several
// writes its sums as they are.
struct W4Range {
  int b0, n;
};
__device__ __forceinline__ W4Range w4_part(W4Args& p, int part, int unit) {
  const int nb = p.K / kBlock;
  if (p.splits <= 1) return W4Range{0, nb};
  const uint32_t units = (nb + unit - 1) / unit, each = units / p.splits, more = units - each * p.splits;
  const int b0 = unit * (part * each + min((uint32_t)part, more));
  const int b1 = min(nb, b0 + unit * (int)(each + ((uint32_t)part < more ? 1u : 0u)));
  p.out32 = p.partial + (int64_t)part * p.x_rows * p.N;
  p.out_stride = p.N;
  p.bias = nullptr;
  return W4Range{b0, b1 - b0};
}

// How the product of one matrix is cut (see w4_gemm_cut).  Parts of K are at most 16 and
// have at most 1024 rows of sums together, or one part.
struct W4Cut {
  int S, tiles, parts;  // tiles of 32 S activation rows by 128 tiles weight rows, parts of K
};
inline int w4_most_parts(int64_t rows) { return rows > 512 ? 1 : (int)(rows <= 64 ? 16 : 1024 / rows); }

// Four neighbouring outputs of a row.
__device__ __forceinline__ void w4_store(const W4Args& p, int64_t row, int n, v4f v) {
  if (p.bias) {
    const uint2 b = *reinterpret_cast<const uint2*>(p.bias + n);
    v[0] += bf16_to_f32(b.x & 0xffffu);
    v[1] += bf16_to_f32(b.x >> 16);
    v[2] += bf16_to_f32(b.y & 0xffffu);
    v[3] += bf16_to_f32(b.y >> 16);
  }
  const int64_t at = row * p.out_stride + n;
  if (p.out32) {
    *reinterpret_cast<float4*>(p.out32 + at) = make_float4(v[0], v[1], v[2], v[3]);
  } else {
    *reinterpret_cast<uint2*>(p.out16 + at) =
        make_uint2((uint32_t)f32_to_bf16_rne(v[0]) | ((uint32_t)f32_to_bf16_rne(v[1]) << 16),
                   (uint32_t)f32_to_bf16_rne(v[2]) | ((uint32_t)f32_to_bf16_rne(v[3]) << 16));
  }
}

}  // namespace moe
