// Residual addition and root-mean-square norm, with the result in bf16, in e4m3
// codes with one scale per 128 columns, or in both.
//
// y = z / sqrt(mean(z^2) + eps) * (w + offset), z = x + residual.  A row is read
// once and stays in registers between the sum of squares and the outputs, so
// the kernel is bound by memory: 2 or 4 bytes a value each for x, residual and
// sum, 2 for out, 1 + 1/32 for the codes.  (8192 rows of 7168, bf16 x, fp32 residual and
// sum, out and codes: 150 us, 5.1 TB/s, a little more than a plain copy reaches; 509 tokens of
// 40 rows of 128: 4.1 us; one row of 7168: 4.2 us, a launch and the two round trips to memory.)
//
// LANES lanes of a 256-thread workgroup share a row, each holding NV pieces of 8
// values (16 bytes of bf16): piece v of the row is lane v % LANES's, so that 16
// neighbouring lanes hold a scale block.  Squares add up in fp32 (a lane's in
// order, then across lanes); where the sum leaves fp32's range the row is
// scaled by a power of two first, which changes no bit of the quotient (but of
// values that the row's largest exceeds 2^126 times: these lose bits, or are 0).
#include <algorithm>

#include "common.h"

namespace moe {

namespace {

constexpr int kNormMaxH = 32768;
constexpr int kNormFewRows = 256;
constexpr float kNormMinEps = 1e-12f;

struct NormArgs {
  const void* x;
  int64_t x_stride;
  const void* residual;
  int64_t residual_stride;
  const uint16_t* weight;
  float weight_offset, eps;
  int64_t rows;
  int H, heads;
  void* sum;
  int64_t sum_stride;
  uint16_t* out;
  int64_t out_stride;
  uint8_t* q;
  float* s;
};

typedef float v8f __attribute__((ext_vector_type(8)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

// The conversion instruction, which keeps NaN: f32_to_bf16_rne rounds one of the largest payloads to a zero.  (Of all
// 2^32 fp32 patterns the others come out as by f32_to_bf16_rne.)
__device__ __forceinline__ uint4 to_bf16x8(const float (&v)[8]) {
  return __builtin_bit_cast(uint4, __builtin_convertvector((v8f{v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]}), v8bf));
}
__device__ __forceinline__ void store8(uint16_t* p, const float (&v)[8]) { *reinterpret_cast<uint4*>(p) = to_bf16x8(v); }
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}

// quant_group8 with a maximum that NaN pass through: a block that holds one has NaN for its scale, and with the finite
// codes of such values reads as NaN.  (By a maximum that passes over them it would read as zeros.)
__device__ __forceinline__ float quant_group8_nan(const float (&v)[8], uint2& codes) {
  float amax = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) amax = __builtin_elementwise_maximum(amax, fabsf(v[i]));
#pragma unroll
  for (int m = 8; m >= 1; m >>= 1) amax = __builtin_elementwise_maximum(amax, __shfl_xor(amax, m, 16));
  const float sc = amax / kE4M3Max;
  codes = make_uint2(quantize4_e4m3(v[0], v[1], v[2], v[3], sc), quantize4_e4m3(v[4], v[5], v[6], v[7], sc));
  return sc;
}

// The sum (or the maximum) over a row's lanes, known to all of them.  `red`
// holds a value per wave; a row of several waves takes the whole workgroup.
template <int LANES, int THREADS, bool MAX>
__device__ __forceinline__ float row_reduce(float v, float* red) {
#pragma unroll
  for (int m = 1; m < (LANES < 64 ? LANES : 64); m <<= 1) {
    const float o = __shfl_xor(v, m);
    v = MAX ? fmaxf(v, o) : v + o;
  }
  if constexpr (LANES > 64) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) v = MAX ? fmaxf(v, red[w]) : v + red[w];
  }
  return v;
}

template <typename XT, typename RT, int LANES, int NV>
__global__ __launch_bounds__(LANES > 256 ? LANES : 256) void add_norm_kernel(NormArgs p) {
  constexpr int kThreads = LANES > 256 ? LANES : 256;
  constexpr int kRows = kThreads / LANES;  // per workgroup and turn
  __shared__ float red[3][kThreads / 64];
  const int lane = threadIdx.x % LANES;
  const int pieces = p.H / 8;
  // Pieces past the row's end load the last one again, unconditionally, so that all loads go out together.
  int at[NV];
  bool in[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    in[i] = lane + LANES * i < pieces;
    at[i] = min(lane + LANES * i, pieces - 1) * 8;
  }
  float w[NV][8];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if (p.weight) {
      load8_f32(p.weight + at[i], w[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) w[i][j] = 1.0f;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) w[i][j] += p.weight_offset;
  }
  // A turn's rows leave together where they share barriers (LANES > 64 is one row a workgroup).
  // (Row numbers of 32 bits: there are less than 2^31 rows and at most 2^16 a turn, and a division of 64 bits is a hundred
  // instructions.)
  for (uint32_t row32 = blockIdx.x * kRows + threadIdx.x / LANES; row32 < (uint32_t)p.rows; row32 += gridDim.x * kRows) {
    const int64_t row = row32, t = p.heads == 1 ? row32 : row32 / (uint32_t)p.heads;
    const int64_t in_token = (row - t * p.heads) * p.H;
    const XT* x = static_cast<const XT*>(p.x) + t * p.x_stride + in_token;
    float z[NV][8];
    float squares = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) load8_f32(x + at[i], z[i]);
    if (p.residual) {
      const RT* r = static_cast<const RT*>(p.residual) + t * p.residual_stride + in_token;
      float a[NV][8];
#pragma unroll
      for (int i = 0; i < NV; ++i) load8_f32(r + at[i], a[i]);
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) z[i][j] += a[i][j];
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) z[i][j] = in[i] ? z[i][j] : 0.0f;
    if (p.sum) {
      RT* sum = static_cast<RT*>(p.sum) + t * p.sum_stride + in_token;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (in[i]) store8(sum + at[i], z[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) squares = __builtin_fmaf(z[i][j], z[i][j], squares);
    squares = row_reduce<LANES, kThreads, false>(squares, red[0]);
    float eps = p.eps;
    const bool wide = !(squares < __builtin_huge_valf());
    if (LANES > 64 ? wide : __any(wide)) {
      float top = 0.0f;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(z[i][j]));
      top = row_reduce<LANES, kThreads, true>(top, red[1]);
      // 2^-e with top below 2^(e + 2): squares then add up to 2^19 at most.
      const int e = wide ? max(0, min((int)(__float_as_uint(top) >> 23) - 127, 126)) : 0;
      const float scale = __uint_as_float((uint32_t)(127 - e) << 23);
      float again = 0.0f;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          z[i][j] *= scale;
          again = __builtin_fmaf(z[i][j], z[i][j], again);
        }
      again = row_reduce<LANES, kThreads, false>(again, red[2]);
      if (wide) squares = again;
      eps = eps * scale * scale;
    }
    const float inv = 1.0f / sqrtf(squares / (float)p.H + eps);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) z[i][j] = z[i][j] * inv * w[i][j];
    if (p.out) {
      uint16_t* out = p.out + t * p.out_stride + in_token;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (in[i]) store8(out + at[i], z[i]);
      }
    }
    if (LANES >= 16 && p.q) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (in[i]) {  // a scale block's 16 lanes together: H is a multiple of 128
          uint2 codes;
          const float sc = quant_group8_nan(z[i], codes);
          *reinterpret_cast<uint2*>(p.q + row * p.H + at[i]) = codes;
          if (at[i] % kBlock == 0) p.s[row * (p.H / kBlock) + at[i] / kBlock] = sc;
        }
      }
    }
    if constexpr (LANES > 64) __syncthreads();  // `red` is written again
  }
}

template <typename XT, typename RT, int LANES, int NV>
void launch_norm(const NormArgs& a, hipStream_t stream) {
  constexpr int kThreads = LANES > 256 ? LANES : 256;
  constexpr int kRows = kThreads / LANES;
  const int64_t blocks = std::min<int64_t>((a.rows + kRows - 1) / kRows, 256 * 2048 / kThreads);
  MOE_LAUNCH("add_norm", (add_norm_kernel<XT, RT, LANES, NV>), dim3((unsigned)blocks), dim3(kThreads), 0, stream, a);
}

template <typename XT, typename RT>
void launch_norm_h(const NormArgs& a, hipStream_t stream) {
  if (a.H <= 64) launch_norm<XT, RT, 8, 1>(a, stream);
  else if (a.H <= 128) launch_norm<XT, RT, 16, 1>(a, stream);
  else if (a.H <= 512) launch_norm<XT, RT, 64, 1>(a, stream);
  else if (a.H <= 2048) launch_norm<XT, RT, 256, 1>(a, stream);
  // A few rows leave most CUs without work: a row's own time counts, and more lanes take less of it (one row of 7168
  // with residual and codes: 4.2 against 5.4 us).
  else if (a.H <= 8192 && a.rows <= kNormFewRows) launch_norm<XT, RT, 1024, 1>(a, stream);
  else if (a.H <= 8192) launch_norm<XT, RT, 256, 4>(a, stream);
  else launch_norm<XT, RT, 1024, 4>(a, stream);
}

}  // namespace

}  // namespace moe

using namespace moe;

extern "C" moe_status_t moe_add_norm(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride,
                                     const uint16_t* weight, int32_t T, int32_t H, moe_norm_cfg_t cfg, void* sum,
                                     int64_t sum_stride, uint16_t* out, int64_t out_stride, uint8_t* q, float* s,
                                     hipStream_t stream) {
  if (T < 0 || H < 1 || cfg.heads < 1)
    return fail(MOE_ERR_INVALID_ARG, "moe_add_norm: T=%d H=%d heads=%d", T, H, cfg.heads);
  if ((cfg.x_type != MOE_BF16 && cfg.x_type != MOE_F32) || (cfg.stream_type != MOE_BF16 && cfg.stream_type != MOE_F32))
    return fail(MOE_ERR_INVALID_ARG, "moe_add_norm: x_type=%d stream_type=%d", cfg.x_type, cfg.stream_type);
  if (!(cfg.eps >= kNormMinEps && cfg.eps < __builtin_huge_valf()) ||
      !(__builtin_fabsf(cfg.weight_offset) < __builtin_huge_valf()))
    return fail(MOE_ERR_INVALID_ARG, "moe_add_norm: eps=%g (at least 1e-12) weight_offset=%g", (double)cfg.eps,
                (double)cfg.weight_offset);
  if (H % 8 || H > kNormMaxH || (q && H % kBlock))
    return fail(MOE_ERR_UNSUPPORTED_SHAPE, "moe_add_norm: H=%d must be a multiple of 8 (of 128 with codes), at most %d", H,
                kNormMaxH);
  const int64_t width = (int64_t)cfg.heads * H;
  if ((int64_t)T * cfg.heads > 0x7fffffff) return fail(MOE_ERR_UNSUPPORTED_SHAPE, "moe_add_norm: T * heads overflows");
  if (T == 0) return MOE_OK;  // (tensors without values may have no address)
  if (!q != !s) return fail(MOE_ERR_INVALID_ARG, "moe_add_norm: q and s come together");
  if (!out && !q) return fail(MOE_ERR_INVALID_ARG, "moe_add_norm: neither out nor q is given");
  if (!x) return fail(MOE_ERR_INVALID_ARG, "moe_add_norm: null pointer");
  const struct {
    const void* p;
    int64_t stride;
    const char* name;
  } rows[] = {{x, x_stride, "x"}, {residual, residual_stride, "residual"}, {sum, sum_stride, "sum"}, {out, out_stride, "out"}};
  for (const auto& r : rows) {
    if (!r.p) continue;
    if (!aligned(r.p, 16)) return fail(MOE_ERR_INVALID_ARG, "moe_add_norm: %s must be 16-byte aligned", r.name);
    if (r.stride < width || r.stride % 8)
      return fail(MOE_ERR_INVALID_ARG, "moe_add_norm: stride %lld of %s must be a multiple of 8, at least %lld",
                  (long long)r.stride, r.name, (long long)width);
  }
  if (!aligned(weight, 16) || !aligned(q, 8) || !aligned(s, 4))
    return fail(MOE_ERR_INVALID_ARG, "moe_add_norm: misaligned pointer");
  NormArgs a{x, x_stride, residual, residual_stride, weight, cfg.weight_offset, cfg.eps, (int64_t)T * cfg.heads, H,
             cfg.heads, sum, sum_stride, out, out_stride, q, s};
  if (cfg.x_type == MOE_BF16) {
    if (cfg.stream_type == MOE_BF16) launch_norm_h<uint16_t, uint16_t>(a, stream);
    else launch_norm_h<uint16_t, float>(a, stream);
  } else {
    if (cfg.stream_type == MOE_BF16) launch_norm_h<float, uint16_t>(a, stream);
    else launch_norm_h<float, float>(a, stream);
  }
  return check_launch("moe_add_norm");
}
