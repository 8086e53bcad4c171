// 4-bit weights: quantization and the packed layout.  Offline, bound by memory.
#include <algorithm>

#include "w4.h"

namespace moe {

namespace {

// One lane a group of 32 columns.  2^e is the smallest power of two with
// max|w| <= 7 * 2^e: with 2^x <= max < 2^(x + 1) that is e = x - 2, or x - 1 where
// the mantissa is above 1.75.  The division by 2^e is exact but for results far
// below the smallest code.  The codes have no NaN and no infinity: a group with one
// gets the scale byte kW4NoScale, which pack_scale_w4_kernel reports.
__global__ __launch_bounds__(256) void quant_weight_w4_kernel(const float* __restrict__ w, int64_t groups,
                                                              uint8_t* __restrict__ q, uint8_t* __restrict__ s) {
  for (int64_t g = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; g < groups; g += (int64_t)gridDim.x * blockDim.x) {
    float v[4][8];
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      load8_f32(w + g * kW4Group + 8 * i, v[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) top = __builtin_elementwise_maximum(top, fabsf(v[i][j]));  // NaN passes through
    }
    const uint32_t bits = __float_as_uint(top);
    int e = (int)(bits >> 23) - 127 - 2 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    e = max(-120, min(e, 120));
    const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
    uint32_t packed[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      packed[i] = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float a = fabsf(v[i][j]) * inv;
        // The borders between neighbouring values; one that lies on a border takes the even code.
        uint32_t c = (a > 0.25f) + (a >= 0.75f) + (a > 1.25f) + (a >= 1.75f) + (a > 2.5f) + (a >= 3.5f) + (a > 5.0f);
        c |= (__float_as_uint(v[i][j]) >> 31) << 3;
        packed[i] |= c << (4 * j);
      }
    }
    *reinterpret_cast<uint4*>(q + g * (kW4Group / 2)) = make_uint4(packed[0], packed[1], packed[2], packed[3]);
    s[g] = (uint8_t)(top < __builtin_huge_valf() ? e + 127 : kW4NoScale);
  }
}

// One thread writes 16 bytes of codes: lane 16 kq + r of tile (g, b), dword j the
// codes of row 16g + r, columns 128b + 32j + 8kq.
__global__ __launch_bounds__(256) void pack_weight_w4_kernel(const uint8_t* __restrict__ q, int64_t pieces, int cols,
                                                             uint8_t* __restrict__ out) {
  const int nb = cols / kBlock;
  for (int64_t c = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; c < pieces; c += (int64_t)gridDim.x * blockDim.x) {
    const int r = (int)(c & 15), kq = (int)((c >> 4) & 3);
    const int64_t tile = c >> 6;
    const int64_t g = tile / nb;
    const int b = (int)(tile - g * nb);
    const uint8_t* src = q + (g * 16 + r) * (int64_t)(cols / 2) + b * (kBlock / 2) + 4 * kq;
    uint32_t d[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) d[j] = *reinterpret_cast<const uint32_t*>(src + 16 * j);
    *reinterpret_cast<uint4*>(out + c * 16) = make_uint4(d[0], d[1], d[2], d[3]);
  }
}

// One thread writes a row's four scales of a 128-column block (or the padding).
__global__ __launch_bounds__(256) void pack_scale_w4_kernel(const uint8_t* __restrict__ s, int64_t words, int cols,
                                                            int chunks, uint8_t* __restrict__ out,
                                                            int32_t* __restrict__ dev_status) {
  const int groups = cols / kW4Group;
  for (int64_t c = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; c < words; c += (int64_t)gridDim.x * blockDim.x) {
    const int i = (int)(c & 3), r = (int)((c >> 2) & 15);
    const int64_t tile = c >> 6;
    const int64_t g = tile / chunks;
    const int at = (int)(tile - g * chunks) * (kW4ScaleCols / kW4Group) + 4 * i;
    uint32_t v = 0x7f7f7f7fu;
    if (at < groups) {
      v = *reinterpret_cast<const uint32_t*>(s + (g * 16 + r) * (int64_t)groups + at);
      bool bad = false;
#pragma unroll
      for (int j = 0; j < 4; ++j) bad |= ((v >> (8 * j)) & 255u) > (uint32_t)kW4MaxScale;
      if (bad && dev_status) atomicOr(dev_status, MOE_DEV_BAD_SCALE);
    }
    *reinterpret_cast<uint32_t*>(out + c * 4) = v;
  }
}

unsigned blocks_for(int64_t threads) { return (unsigned)std::min<int64_t>((threads + 255) / 256, 1 << 16); }

}  // namespace

}  // namespace moe

using namespace moe;

extern "C" moe_status_t moe_quant_weight_w4(const float* w, int32_t n_mats, int32_t rows, int32_t cols, uint8_t* q,
                                            uint8_t* s, hipStream_t stream) {
  if (n_mats < 0 || rows <= 0 || cols <= 0)
    return fail(MOE_ERR_INVALID_ARG, "moe_quant_weight_w4: n_mats=%d rows=%d cols=%d", n_mats, rows, cols);
  if (cols % kW4Group)
    return fail(MOE_ERR_UNSUPPORTED_SHAPE, "moe_quant_weight_w4: cols=%d not a multiple of %d", cols, kW4Group);
  if (n_mats == 0) return MOE_OK;
  if (!w || !q || !s) return fail(MOE_ERR_INVALID_ARG, "moe_quant_weight_w4: null pointer");
  if (!aligned(w, 16) || !aligned(q, 16)) return fail(MOE_ERR_INVALID_ARG, "moe_quant_weight_w4: misaligned pointer");
  const int64_t rows_all = (int64_t)n_mats * rows;
  if (rows_all > (INT64_MAX >> 3) / cols) return fail(MOE_ERR_UNSUPPORTED_SHAPE, "moe_quant_weight_w4: too many weights");
  const int64_t groups = rows_all * (cols / kW4Group);
  MOE_LAUNCH("quant_weight_w4", quant_weight_w4_kernel, dim3(blocks_for(groups)), dim3(256), 0, stream, w, groups, q, s);
  return check_launch("moe_quant_weight_w4");
}

extern "C" size_t moe_w4_scale_bytes(int32_t n_mats, int32_t rows, int32_t cols) {
  if (n_mats <= 0 || rows <= 0 || cols <= 0 || rows % 16 || cols % kBlock) return 0;
  return (size_t)n_mats * (size_t)(rows / 16) * (size_t)w4_scale_chunks(cols) * kW4ScaleTile;
}

extern "C" moe_status_t moe_pack_weight_w4(const uint8_t* q, const uint8_t* s, int32_t n_mats, int32_t rows, int32_t cols,
                                           uint8_t* packed, uint8_t* packed_s, int32_t* dev_status, hipStream_t stream) {
  if (n_mats < 0 || rows <= 0 || cols <= 0)
    return fail(MOE_ERR_INVALID_ARG, "moe_pack_weight_w4: n_mats=%d rows=%d cols=%d", n_mats, rows, cols);
  if (rows % 16 || cols % kBlock)
    return fail(MOE_ERR_UNSUPPORTED_SHAPE, "moe_pack_weight_w4: %dx%d (rows a multiple of 16, cols of 128)", rows, cols);
  if (n_mats == 0) return MOE_OK;
  if (!q || !s || !packed || !packed_s) return fail(MOE_ERR_INVALID_ARG, "moe_pack_weight_w4: null pointer");
  if (!aligned(q, 16) || !aligned(s, 4) || !aligned(packed, 16) || !aligned(packed_s, 16) || !aligned(dev_status, 4))
    return fail(MOE_ERR_INVALID_ARG, "moe_pack_weight_w4: misaligned pointer");
  const int64_t rows_all = (int64_t)n_mats * rows;
  if (rows_all > (INT64_MAX >> 3) / cols) return fail(MOE_ERR_UNSUPPORTED_SHAPE, "moe_pack_weight_w4: too many weights");
  const int64_t pieces = rows_all * (cols / kW4Group);
  MOE_LAUNCH("pack_weight_w4", pack_weight_w4_kernel, dim3(blocks_for(pieces)), dim3(256), 0, stream, q, pieces, cols, packed);
  moe_status_t st = check_launch("moe_pack_weight_w4");
  if (st != MOE_OK) return st;
  const int64_t words = (int64_t)(moe_w4_scale_bytes(1, 16, cols) / 4) * (rows_all / 16);
  MOE_LAUNCH("pack_scale_w4", pack_scale_w4_kernel, dim3(blocks_for(words)), dim3(256), 0, stream, s, words, cols,
             (int)w4_scale_chunks(cols), packed_s, dev_status);
  return check_launch("moe_pack_weight_w4");
}
