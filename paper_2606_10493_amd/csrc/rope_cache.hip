// Rotary positions, the quantized key/value cache's write and its read.
//
// All three are bound by memory: a head's row is one group of head_dim / 8
// lanes with 8 elements each (16 bytes of bf16, 8 bytes of codes), so every
// row moves in whole 64- to 256-byte pieces.  8192 tokens of 32 + 2 * 8 heads of
// 128: 47 us for 204 MB, 4.3 TB/s, and 104k cached tokens read back: 123 us for 643
// MB, 5.2 TB/s, where a copy of 4 GiB reaches 4.8.  A step of 16 tokens takes 4 us,
// what a launch and three dependent reads take.
#include <math.h>

#include <algorithm>

#include "attention.h"

namespace moe {

namespace {

// ----------------------------------------------------------------- the table
// One thread per (position, pair): frequency, angle, cosine and sine in 64
// bits.  Positions go to millions and an fp32 angle p * f has lost its last
// digits long before (2^-24 of 10^6 turns is a tenth of a radian).
__global__ __launch_bounds__(256) void rope_table_kernel(moe_rope_cfg_t cfg, int64_t n, float* __restrict__ table) {
  const int half = cfg.rot_dim / 2;
  const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (idx >= n) return;
  const int64_t p = idx / half;
  const int i = (int)(idx - p * half);
  const double g = pow(cfg.base, -2.0 * i / cfg.rot_dim);
  double f = g;
  if (cfg.scaling == MOE_ROPE_LINEAR) f = g / cfg.factor;
  if (cfg.scaling == MOE_ROPE_BY_PARTS) {
    const double turns = cfg.original_len * g / 6.283185307179586476925;
    const double w = fmin(fmax((turns - cfg.slow_turns) / (cfg.fast_turns - cfg.slow_turns), 0.0), 1.0);
    f = (1.0 - w) * g / cfg.factor + w * g;
  }
  const double a = (double)p * f;
  table[p * cfg.rot_dim + i] = (float)(cos(a) * cfg.magnitude);
  table[p * cfg.rot_dim + half + i] = (float)(sin(a) * cfg.magnitude);
}

// ------------------------------------------------------------ rotate and write
struct RopeArgs {
  const uint16_t *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;
  const int32_t *positions, *slots;
  const float* table;
  moe_kv_cache_t cache;
  uint16_t *q_out, *k_out;  // may be q, k: a lane reads what it writes before that, and nothing else
  int32_t* status;
  int32_t n_pos, rot_dim, page_shift;
  int T, q_heads, kv_heads, layout;
};

// Eight elements at offset e of a head's row, rotated.  c, s: this lane's cosines
// and sines: HALF 8 + 8 (its elements' pairs), INTERLEAVED 4 + 4.  partner: HALF,
// the elements that lie half the rotated part away.  The definition rounds every
// product and sum: no FMA.
__device__ __forceinline__ void rotate8(float (&x)[8], const uint4 partner, bool interleaved, bool low,
                                        const float (&c)[8], const float (&s)[8]) {
#pragma clang fp contract(off)
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float a = x[2 * i], b = x[2 * i + 1];
      const float ac = a * c[i], bs = b * s[i], bc = b * c[i], as = a * s[i];
      x[2 * i] = ac - bs;
      x[2 * i + 1] = bc + as;
    }
    return;
  }
  float p[8];
  bf16x8_to_f32(partner, p);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float xc = x[i] * c[i], ps = p[i] * s[i];
    x[i] = low ? xc - ps : xc + ps;
  }
}

__device__ __forceinline__ uint4 to_bf16x8(const float (&x)[8]) {
  return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}

// A group of D / 8 lanes takes one token's rows PER * blockIdx.y .. + PER - 1,
// counted over the query heads, the key heads and (with a cache) the value
// heads.  The groups of a wave are consecutive tokens at the same rows, so a
// wave's branches go one way.  Rows share the token's position, slot and table
// row: four a group where that leaves the card 4096 workgroups (8192 tokens, 48
// rows: 61 us with one a group, 48 with four), else one (16 tokens: 4.0 us, 6.4
// with four).
template <int D, int PER>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  constexpr int kLanes = D / 8, kTokens = 256 / kLanes;
  const int sub = threadIdx.x % kLanes, e = sub * 8;
  const int64_t t = (int64_t)blockIdx.x * kTokens + threadIdx.x / kLanes;
  if (t >= a.T) return;  // whole groups leave together
  const int n_rows = a.q_heads + a.kv_heads + (a.slots ? a.kv_heads : 0);
  const bool interleaved = a.layout == MOE_ROPE_INTERLEAVED;

  int pos = a.positions[t];
  if (pos < 0 || pos >= a.n_pos) {
    if (a.status && sub == 0) atomicOr(a.status, MOE_DEV_BAD_POSITION);
    pos = 0;
  }
  float c[8] = {}, s[8] = {};
  if (e < a.rot_dim) {
    const int half = a.rot_dim / 2;
    const float* row = a.table + (int64_t)pos * a.rot_dim + (interleaved ? e / 2 : e < half ? e : e - half);
    if (interleaved) {
      const float4 x = *reinterpret_cast<const float4*>(row), y = *reinterpret_cast<const float4*>(row + half);
      c[0] = x.x; c[1] = x.y; c[2] = x.z; c[3] = x.w;
      s[0] = y.x; s[1] = y.y; s[2] = y.z; s[3] = y.w;
    } else {
      load8_f32(row, c);
      load8_f32(row + half, s);
    }
  }
  int64_t page = -1;
  int at = 0;
  if (a.slots) {
    const int slot = a.slots[t];
    page = slot >> a.page_shift;  // a negative slot stays negative
    at = slot & (a.cache.page_size - 1);
    if (page >= a.cache.n_pages) {
      if (a.status && sub == 0) atomicOr(a.status, MOE_DEV_BAD_SLOT);
      page = -1;
    }
  }

  const int half = a.rot_dim / 2;
  const bool turns = e < a.rot_dim, low = e < half;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int r = blockIdx.y * PER + j;
    if (r >= n_rows) break;
    const int kind = r < a.q_heads ? 0 : r < a.q_heads + a.kv_heads ? 1 : 2;
    const int h = kind == 0 ? r : kind == 1 ? r - a.q_heads : r - a.q_heads - a.kv_heads;
    const uint16_t* base = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
    if (!base) continue;
    const uint16_t* row = base + t * (kind == 0 ? a.q_stride : kind == 1 ? a.k_stride : a.v_stride) + h * D;
    float x[8];
    const uint4 raw = *reinterpret_cast<const uint4*>(row + e);
    uint4 partner = raw;  // HALF: what the lane half the rotated part away has
    if (kind < 2 && !interleaved) {
      const int from = !turns ? sub : low ? sub + half / 8 : sub - half / 8;
      partner = make_uint4(__shfl(raw.x, from, kLanes), __shfl(raw.y, from, kLanes), __shfl(raw.z, from, kLanes),
                           __shfl(raw.w, from, kLanes));
    }
    bf16x8_to_f32(raw, x);
    if (kind < 2 && turns) rotate8(x, partner, interleaved, low, c, s);
    if (kind == 0) *reinterpret_cast<uint4*>(a.q_out + (t * a.q_heads + h) * D + e) = to_bf16x8(x);
    if (kind == 1 && a.k_out) *reinterpret_cast<uint4*>(a.k_out + (t * a.kv_heads + h) * D + e) = to_bf16x8(x);
    if (kind > 0 && page >= 0) {
      float amax = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(x[i]));
#pragma unroll
      for (int m = kLanes / 2; m >= 1; m >>= 1) amax = fmaxf(amax, __shfl_xor(amax, m, kLanes));
      const float sc = amax / kE4M3Max;
      const int64_t place = ((page * a.kv_heads + h) << a.page_shift) + at;
      uint8_t* codes = kind == 1 ? a.cache.k : a.cache.v;
      *reinterpret_cast<uint2*>(codes + place * D + e) =
          make_uint2(quantize4_e4m3(x[0], x[1], x[2], x[3], sc), quantize4_e4m3(x[4], x[5], x[6], x[7], sc));
      if (sub == 0) (kind == 1 ? a.cache.k_scale : a.cache.v_scale)[place] = sc;
    }
  }
}

constexpr int64_t kSpanTokens = 1 << 26;  // tokens per launch: a grid's side has less than 2^32 threads

template <int D>
moe_status_t launch_rope(const RopeArgs& all, const char* name, hipStream_t stream) {
  const int n_rows = all.q_heads + all.kv_heads + (all.slots ? all.kv_heads : 0);
  for (int64_t t0 = 0; t0 < all.T; t0 += kSpanTokens) {
    RopeArgs a = all;
    a.T = (int)std::min<int64_t>(kSpanTokens, all.T - t0);
    if (a.q) { a.q += t0 * a.q_stride; a.q_out += t0 * a.q_heads * D; }
    if (a.k) a.k += t0 * a.k_stride;
    if (a.k_out) a.k_out += t0 * a.kv_heads * D;
    if (a.v) a.v += t0 * a.v_stride;
    a.positions += t0;
    if (a.slots) a.slots += t0;
    const unsigned gx = (unsigned)((a.T + 256 / (D / 8) - 1) / (256 / (D / 8)));
    if ((int64_t)gx * n_rows < 4096)
      MOE_LAUNCH(name, (rope_kernel<D, 1>), dim3(gx, n_rows), dim3(256), 0, stream, a);
    else
      MOE_LAUNCH(name, (rope_kernel<D, 4>), dim3(gx, (n_rows + 3) / 4), dim3(256), 0, stream, a);
  }
  return check_launch(name);
}

moe_status_t check_rope(const moe_attn_dims_t& d, int32_t T, const int32_t* positions, const float* table, int32_t n_pos,
                        int32_t rot_dim, moe_rope_layout_t layout, const char* who) {
  const moe_status_t st = check_attn_dims(d, who);
  if (st != MOE_OK) return st;
  if (T < 0 || n_pos < 1) return fail(MOE_ERR_INVALID_ARG, "%s: T=%d n_pos=%d", who, T, n_pos);
  if (layout != MOE_ROPE_HALF && layout != MOE_ROPE_INTERLEAVED)
    return fail(MOE_ERR_INVALID_ARG, "%s: layout=%d", who, (int)layout);
  if (rot_dim < 16 || rot_dim % 16 || rot_dim > d.head_dim)
    return fail(MOE_ERR_UNSUPPORTED_SHAPE, "%s: rot_dim=%d must be a multiple of 16, 16..%d", who, rot_dim, d.head_dim);
  if (T > 0 && (!positions || !table || !aligned(table, 16)))
    return fail(MOE_ERR_INVALID_ARG, "%s: positions or table NULL, or table not 16-byte aligned", who);
  return MOE_OK;
}

// ------------------------------------------------------------------ read back
// The sequence of token t: cu[lo] <= t < cu[lo + 1], cu[0] <= t < cu[B].  The
// group's lanes look at as many places at once as they are, so that up to 17 (9)
// sequences cost one round trip and 289 (81) two.  Offsets that decrease give
// some lo in [0, B).
template <int kLanes>
__device__ __forceinline__ int sequence_of(const int32_t* __restrict__ cu, int B, int64_t t, int sub) {
  int lo = 0, hi = B;
  while (hi - lo > 1) {
    const int hop = (hi - lo + kLanes) / (kLanes + 1), probe = lo + (sub + 1) * hop;
    const uint64_t below = __ballot(probe < hi && cu[min(probe, B)] <= t);
    const int n = __popcll(below >> ((threadIdx.x & 63) - sub) & ((1u << kLanes) - 1));
    lo += n * hop;
    hi = min(hi, lo + hop);
  }
  return min(lo, B - 1);
}

// A group of D / 8 lanes takes one token's keys and values of `per` heads.  With a
// status word the grid has one column of workgroups more, the first of which looks
// at the offsets: those of a sequence that the cut leaves nothing, too.  What
// is written is read by another launch, if at all from a cache that holds all of
// it: the stores are non-temporal (104k tokens of 8 heads of 128: 132 -> 123 us).
template <int D>
__global__ __launch_bounds__(256) void cache_read_kernel(moe_kv_cache_t cache, int page_shift, int kv_heads, int per,
                                                         const int32_t* __restrict__ pages, int B, int width,
                                                         const int32_t* __restrict__ cu, int T,
                                                         uint16_t* __restrict__ k_out, uint16_t* __restrict__ v_out,
                                                         int32_t* status, uint32_t looks) {
  constexpr int kLanes = D / 8, kTokens = 256 / kLanes;
  const int sub = threadIdx.x % kLanes;
  if (blockIdx.x == looks) {
    if (blockIdx.y > 0) return;
    bool cut = false;
    for (int64_t i = threadIdx.x; i < B; i += 256) cut |= cu[i] < 0 || cu[i + 1] > T || cu[i] > cu[i + 1];
    if (__any(cut) && threadIdx.x % 64 == 0) atomicOr(status, MOE_DEV_BAD_LENGTH);
    return;
  }
  const int64_t t = (int64_t)blockIdx.x * kTokens + threadIdx.x / kLanes;
  if (t >= T || t < cu[0] || t >= cu[B]) return;  // whole groups leave together
  const int b = sequence_of<kLanes>(cu, B, t, sub);
  const int64_t at = t - cu[b];
  int bad = 0;
  int64_t page = 0;
  if (at < 0 || (at >> page_shift) >= width) {
    bad = MOE_DEV_BAD_LENGTH;
  } else {
    page = pages[(int64_t)b * width + (at >> page_shift)];
    if (page < 0 || page >= cache.n_pages) bad = MOE_DEV_BAD_PAGE;
  }
  if (bad && status && sub == 0) atomicOr(status, bad);
  const int64_t place0 = ((page * kv_heads) << page_shift) + (at & (cache.page_size - 1));
  const int h1 = min((int)(blockIdx.y + 1) * per, kv_heads);
#pragma unroll 4
  for (int h = blockIdx.y * per; h < h1; ++h) {
    const int64_t place = place0 + ((int64_t)h << page_shift);
    const int64_t out = (t * kv_heads + h) * D + sub * 8;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      uint4 o = make_uint4(0, 0, 0, 0);
      if (!bad) {
        const uint2 codes = *reinterpret_cast<const uint2*>((w ? cache.v : cache.k) + place * D + sub * 8);
        const float s = (w ? cache.v_scale : cache.k_scale)[place];
        const v8bf y = e4m3x8_to_bf16(codes.x, codes.y);
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)y[i] * s;
        o = to_bf16x8(x);
      }
      const u32x4_stream words = {o.x, o.y, o.z, o.w};
      __builtin_nontemporal_store(words, reinterpret_cast<u32x4_stream*>((w ? v_out : k_out) + out));
    }
  }
}

int log2_of(int x) { return __builtin_ctz((unsigned)x); }

}  // namespace

}  // namespace moe

using namespace moe;

extern "C" moe_status_t moe_rope_table(moe_rope_cfg_t cfg, int32_t n_pos, float* table, hipStream_t stream) {
  if (cfg.rot_dim < 16 || cfg.rot_dim % 16 || cfg.rot_dim > 128)
    return fail(MOE_ERR_UNSUPPORTED_SHAPE, "moe_rope_table: rot_dim=%d must be a multiple of 16, 16..128", cfg.rot_dim);
  const bool scaled = cfg.scaling == MOE_ROPE_LINEAR || cfg.scaling == MOE_ROPE_BY_PARTS;
  if (n_pos < 0 || (cfg.scaling != MOE_ROPE_PLAIN && !scaled) || !(cfg.base > 1.0) || !isfinite(cfg.base) ||
      !isfinite(cfg.magnitude) || (scaled && (!(cfg.factor > 0.0) || !isfinite(cfg.factor))) ||
      (cfg.scaling == MOE_ROPE_BY_PARTS && (!(cfg.original_len > 0.0) || !isfinite(cfg.original_len) ||
                                            !(cfg.slow_turns >= 0.0) || !(cfg.fast_turns > cfg.slow_turns) ||
                                            !isfinite(cfg.fast_turns))))
    return fail(MOE_ERR_INVALID_ARG,
                "moe_rope_table: n_pos=%d scaling=%d base=%g factor=%g original_len=%g turns %g..%g magnitude=%g", n_pos,
                cfg.scaling, cfg.base, cfg.factor, cfg.original_len, cfg.slow_turns, cfg.fast_turns, cfg.magnitude);
  if (n_pos == 0) return MOE_OK;
  if (!table || !aligned(table, 16)) return fail(MOE_ERR_INVALID_ARG, "moe_rope_table: table NULL or not 16-byte aligned");
  const int half = cfg.rot_dim / 2;
  constexpr int64_t kSpan = 1 << 22;  // positions per launch: less than 2^32 threads
  if (n_pos > kSpan) return fail(MOE_ERR_UNSUPPORTED_SHAPE, "moe_rope_table: n_pos=%d is over %lld", n_pos, (long long)kSpan);
  const int64_t n = (int64_t)n_pos * half;
  MOE_LAUNCH("rope_table", rope_table_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, stream, cfg, n, table);
  return check_launch("moe_rope_table");
}

extern "C" moe_status_t moe_rope(moe_attn_dims_t d, int32_t T, const uint16_t* q, int64_t q_stride, const uint16_t* k,
                                 int64_t k_stride, const int32_t* positions, const float* table, int32_t n_pos,
                                 int32_t rot_dim, moe_rope_layout_t layout, uint16_t* q_out, uint16_t* k_out,
                                 int32_t* dev_status, hipStream_t stream) {
  moe_status_t st = check_rope(d, T, positions, table, n_pos, rot_dim, layout, "moe_rope");
  if (st != MOE_OK || T == 0) return st;
  if (!q != !q_out || !k != !k_out || (!q && !k))
    return fail(MOE_ERR_INVALID_ARG, "moe_rope: q and q_out, and k and k_out, are given together, one pair at least");
  if (q && (st = check_rows(q, q_stride, d.q_heads, d.head_dim, "moe_rope", "q")) != MOE_OK) return st;
  if (k && (st = check_rows(k, k_stride, d.kv_heads, d.head_dim, "moe_rope", "k")) != MOE_OK) return st;
  if (!aligned(q_out, 16) || !aligned(k_out, 16))
    return fail(MOE_ERR_INVALID_ARG, "moe_rope: outputs must be 16-byte aligned");
  if ((q == q_out && q && q_stride != (int64_t)d.q_heads * d.head_dim) ||
      (k == k_out && k && k_stride != (int64_t)d.kv_heads * d.head_dim))
    return fail(MOE_ERR_INVALID_ARG, "moe_rope: in place needs contiguous rows");
  RopeArgs a{q, k, nullptr, q_stride, k_stride, 0, positions, nullptr, table, moe_kv_cache_t{}, q_out, k_out,
             dev_status, n_pos, rot_dim, 0, T, d.q_heads, d.kv_heads, (int)layout};
  return d.head_dim == 64 ? launch_rope<64>(a, "rope", stream) : launch_rope<128>(a, "rope", stream);
}

extern "C" moe_status_t moe_rope_cache(moe_attn_dims_t d, int32_t T, const uint16_t* q, int64_t q_stride,
                                       const uint16_t* k, int64_t k_stride, const uint16_t* v, int64_t v_stride,
                                       const int32_t* positions, const float* table, int32_t n_pos, int32_t rot_dim,
                                       moe_rope_layout_t layout, const int32_t* slots, moe_kv_cache_t cache,
                                       uint16_t* q_out, uint16_t* k_out, int32_t* dev_status, hipStream_t stream) {
  moe_status_t st = check_rope(d, T, positions, table, n_pos, rot_dim, layout, "moe_rope_cache");
  if (st != MOE_OK) return st;
  if ((st = check_cache(cache, "moe_rope_cache")) != MOE_OK) return st;
  if (T == 0) return MOE_OK;
  if ((st = check_rows(q, q_stride, d.q_heads, d.head_dim, "moe_rope_cache", "q")) != MOE_OK) return st;
  if ((st = check_rows(k, k_stride, d.kv_heads, d.head_dim, "moe_rope_cache", "k")) != MOE_OK) return st;
  if ((st = check_rows(v, v_stride, d.kv_heads, d.head_dim, "moe_rope_cache", "v")) != MOE_OK) return st;
  if (!slots || !q_out) return fail(MOE_ERR_INVALID_ARG, "moe_rope_cache: slots or q_out is NULL");
  if (!aligned(q_out, 16) || !aligned(k_out, 16))
    return fail(MOE_ERR_INVALID_ARG, "moe_rope_cache: outputs must be 16-byte aligned");
  if ((q == q_out && q_stride != (int64_t)d.q_heads * d.head_dim) ||
      (k == k_out && k_stride != (int64_t)d.kv_heads * d.head_dim))
    return fail(MOE_ERR_INVALID_ARG, "moe_rope_cache: in place needs contiguous rows");
  RopeArgs a{q, k, v, q_stride, k_stride, v_stride, positions, slots, table, cache, q_out, k_out,
             dev_status, n_pos, rot_dim, log2_of(cache.page_size), T, d.q_heads, d.kv_heads, (int)layout};
  return d.head_dim == 64 ? launch_rope<64>(a, "rope_cache", stream) : launch_rope<128>(a, "rope_cache", stream);
}

extern "C" moe_status_t moe_cache_read(moe_attn_dims_t d, moe_kv_cache_t cache, const int32_t* page_table, int32_t B,
                                       int32_t table_width, const int32_t* cu, int32_t T, uint16_t* k_out,
                                       uint16_t* v_out, int32_t* dev_status, hipStream_t stream) {
  moe_status_t st = check_attn_dims(d, "moe_cache_read");
  if (st != MOE_OK) return st;
  if ((st = check_cache(cache, "moe_cache_read")) != MOE_OK) return st;
  if (B < 0 || T < 0 || table_width < 0)
    return fail(MOE_ERR_INVALID_ARG, "moe_cache_read: B=%d T=%d table_width=%d", B, T, table_width);
  if (B == 0 || T == 0) return MOE_OK;
  if ((!page_table && table_width > 0) || !cu || !k_out || !v_out) return fail(MOE_ERR_INVALID_ARG, "moe_cache_read: null pointer");
  if (!aligned(k_out, 16) || !aligned(v_out, 16))
    return fail(MOE_ERR_INVALID_ARG, "moe_cache_read: outputs must be 16-byte aligned");
  const int shift = log2_of(cache.page_size), per = 256 / (d.head_dim / 8);
  if (T > kSpanTokens) return fail(MOE_ERR_UNSUPPORTED_SHAPE, "moe_cache_read: T=%d is over %lld", T, (long long)kSpanTokens);
  const unsigned gx = (unsigned)((T + per - 1) / per);
  const int heads = gx < 1024 ? 1 : d.kv_heads;  // few tokens: more workgroups rather than longer ones
  const uint32_t looks = dev_status ? gx : ~0u;  // the column that looks at the offsets
  const dim3 grid(gx + (dev_status ? 1 : 0), (d.kv_heads + heads - 1) / heads);
  if (d.head_dim == 64)
    MOE_LAUNCH("cache_read", cache_read_kernel<64>, grid, dim3(256), 0, stream, cache, shift, d.kv_heads, heads,
               page_table, B,
               table_width, cu, T, k_out, v_out, dev_status, looks);
  else
    MOE_LAUNCH("cache_read", cache_read_kernel<128>, grid, dim3(256), 0, stream, cache, shift, d.kv_heads, heads,
               page_table, B,
               table_width, cu, T, k_out, v_out, dev_status, looks);
  return check_launch("moe_cache_read");
}
