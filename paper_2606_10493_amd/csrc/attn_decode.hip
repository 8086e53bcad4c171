// Attention of one token per sequence over the paged e4m3 cache, behind a
// prefix that all sequences share.
//
// The query heads of a key/value head are the columns of 16x16x32 MFMAs, so a
// key's codes are read and converted once for all of them.  A sequence's own keys
// have its G query heads as columns, the prefix's keys those of all sequences
// (B * G columns), so the prefix is read once for the batch.
//   S^T = K Q^T   (bf16) keys' codes go from the pages to registers as the
//                 first operand (lane: key lane % 16, 16 codes at 16 (lane / 16)
//                 of each 64), converted exactly; a lane ends with the scores of
//                 query lane % 16 for keys 4 (lane / 16) + i
//   O^T = V^T P^T (f16) values' codes go through LDS and come back transposed
//                 (ds_read_b64_tr_b8) in the order of keys that the scores have
// Scales stay fp32: a key's multiplies its score, a value's its numerator.  The
// numerators are rounded once for the product, to f16: a code is exact in f16 as
// it is in bf16, and f16 has three bits more.  Its range is kept by dividing the
// values' scales by their running maximum (`vref`), which rescales the
// accumulator as the running maximum of the scores does; what underflows is
// below 2^-25 of the largest term.
//
// Bound by memory: head_dim + 4 bytes per key, value and head against 4 * G *
// head_dim flops.  One long context has few rows, so keys are cut into parts, one
// workgroup each, whose waves take every fourth step of 32 keys; a second launch
// joins the parts.
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
  float* part_o;   // [B * q_heads][slots][D]: a part's sums, not divided
  float* part_ml;  // [B * q_heads][slots][2]: its running maximum and sum
  int32_t* status;
  int B, width, prefix_len, kv_heads, group, page_shift;
  int part_keys, prefix_parts, own_parts;  // slots: the prefix's parts, then a sequence's own
  int prefix_blocks, own_blocks;           // column blocks of all sequences' and of one's queries
  float c;                                 // scale * log2(e)
};

constexpr int kKeys = 32;  // keys per step of a wave
constexpr int kWaves = 4;
constexpr int kStride = kKeys * kWaves;
constexpr int kMostKeys = 1 << 30;  // of a sequence: key indices and the steps behind them stay in 32 bits

typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));

__device__ __forceinline__ v8h e4m3x8_to_f16(uint32_t lo, uint32_t hi) {
  union {
    v8h v;
    v2h p[4];
  } r;
  r.p[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false);
  r.p[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
  r.p[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false);
  r.p[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
  return r.v;
}

// The running softmax of NC blocks of 16 queries; a lane's query is column
// lane % 16 of each block.
template <int D, int NC>
struct Running {
  v4f o[NC][D / 16];     // O^T / vref: rows 16 i + 4 (lane / 16) + 0..3
  float m[NC], l[NC];    // l: this lane's keys only, summed over the lane groups at the end
  float vref;
};

// The maximum over the four lanes that hold one query (lane, lane ^ 16, ^ 32,
// ^ 48), by register swaps between rows of 16 and of 32 lanes.
__device__ __forceinline__ float quad_max(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// 32 keys and values on their way: lane l has 16-byte chunk l % (D / 16) of rows
// l / (D / 16) + ..., so that a load covers whole rows, and key l's scale (lanes
// 0..31) or value l - 32's.
template <int D>
struct Tile {
  u32x4_stream k[D / 32], v[D / 32];
  float scale;
};

// A part of one sequence's (or the prefix's) keys: [begin, end) of the `len`
// that the `width` entries of `pages` hold, key/value head kvh.
struct Part {
  const int32_t* pages;
  int width, len, begin, end, kvh;
};

// The pages of keys [t, t + 32): each half of 16 lies in one.  Entries behind the
// sequence's last page may be looked at, and are not used.
struct Pages {
  int id[2];
};
__device__ __forceinline__ Pages pages_of(const DecodeArgs& a, const Part& p, int t) {
  Pages r;
#pragma unroll
  for (int u = 0; u < 2; ++u) r.id[u] = p.pages[min((t + 16 * u) >> a.page_shift, p.width - 1)];
  return r;
}

// A wave's part of LDS: keys, values (rows of D codes in 16-byte chunks), scales.
// The swizzles spread what one instruction reads over the 256 bytes of the banks:
// 16 keys at one chunk, or the 16 values' rows of two 8 x 16 blocks at one chunk.
template <int D>
struct Staged {
  static constexpr int kV = kKeys * D, kScale = 2 * kKeys * D, kBytes = kScale + 64 * 4;
  static __device__ __forceinline__ int key(int row, int c) {
    return row * D + ((c ^ (D == 128 ? (row >> 1) & 7 : (row >> 2) & 3)) * 16);
  }
  static __device__ __forceinline__ int value(int row, int c) {
    return kV + row * D + ((c ^ (D == 128 ? ((row >> 1) & 3) | ((row >> 2) & 4) : ((row >> 2) & 1) | ((row >> 3) & 2))) * 16);
  }
};

// Loads keys [t0, t0 + 32), t0 < len.  Keys behind the end repeat the last, or
// the first half where the second holds none.  kOnce: nothing else reads them in
// this launch, so they need no place in the caches (64 ragged contexts: 90 us
// without, 78 with, whole rows per load in both).
template <int D, bool kOnce>
__device__ __forceinline__ void load_tile(const DecodeArgs& a, const Part& p, int t0, const Pages& pg, bool& bad,
                                          Tile<D>& x) {
  constexpr int kChunks = D / 16;
  const int lane = threadIdx.x & 63, mask = a.cache.page_size - 1, last = p.len - 1;
  const bool two = t0 + 16 <= last;
  const int id0 = pg.id[0], id1 = two ? pg.id[1] : id0;
  const bool wrong0 = id0 < 0 || id0 >= a.cache.n_pages, wrong1 = id1 < 0 || id1 >= a.cache.n_pages;
  bad |= wrong0 | wrong1;
  // the first key of each half, counted in rows of the cache
  const int64_t row0 = (((int64_t)(wrong0 ? 0 : id0) * a.kv_heads + p.kvh) << a.page_shift) + (t0 & mask);
  const int64_t row1 = two ? (((int64_t)(wrong1 ? 0 : id1) * a.kv_heads + p.kvh) << a.page_shift) + ((t0 + 16) & mask) : row0;
  const int left = last - t0, left1 = two ? left - 16 : left;  // rows behind these repeat them
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    const int at = 64 * i + lane, row = at / kChunks, c = at % kChunks;
    const int64_t from = (row < 16 ? row0 + min(row, left) : row1 + min(row - 16, left1)) * D + 16 * c;
    const u32x4_stream* k = reinterpret_cast<const u32x4_stream*>(a.cache.k + from);
    const u32x4_stream* v = reinterpret_cast<const u32x4_stream*>(a.cache.v + from);
    x.k[i] = kOnce ? __builtin_nontemporal_load(k) : *k;
    x.v[i] = kOnce ? __builtin_nontemporal_load(v) : *v;
  }
  const int row = lane & 31;
  const float* scales = lane < 32 ? a.cache.k_scale : a.cache.v_scale;
  x.scale = scales[row < 16 ? row0 + min(row, left) : row1 + min(row - 16, left1)];
}

// The step at t0, whose keys and values are in x; once they are in LDS, `next`
// loads those of the next step.
template <int D, int NC, typename Next>
__device__ __forceinline__ void use_tile(const DecodeArgs& a, const Part& p, int t0, const Tile<D>& x,
                                         const v8bf (&qf)[NC][D / 32], uint8_t* lds, Running<D, NC>& run, Next next) {
  constexpr int kChunks = D / 16;
  const int lane = threadIdx.x & 63, g = lane >> 4, c16 = lane & 15;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    const int at = 64 * i + lane;
    *reinterpret_cast<u32x4_stream*>(lds + Staged<D>::key(at / kChunks, at % kChunks)) = x.k[i];
    *reinterpret_cast<u32x4_stream*>(lds + Staged<D>::value(at / kChunks, at % kChunks)) = x.v[i];
  }
  *reinterpret_cast<float*>(lds + Staged<D>::kScale + 4 * lane) = x.scale;
  next();
  v4f s[NC][2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
#pragma unroll
    for (int n = 0; n < NC; ++n) s[n][u] = v4f{};
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      const uint4 k = *reinterpret_cast<const uint4*>(lds + Staged<D>::key(16 * u + c16, g + 4 * i));
      const v8bf lo = e4m3x8_to_bf16(k.x, k.y), hi = e4m3x8_to_bf16(k.z, k.w);
#pragma unroll
      for (int n = 0; n < NC; ++n) {
        s[n][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lo, qf[n][2 * i], s[n][u], 0, 0, 0);
        s[n][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi, qf[n][2 * i + 1], s[n][u], 0, 0, 0);
      }
    }
  }
  float ks[2][4], vs[2][4];
  float vtop = run.vref;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const v4f kk = *reinterpret_cast<const v4f*>(lds + Staged<D>::kScale + 4 * (16 * u + 4 * g));
    const v4f vv = *reinterpret_cast<const v4f*>(lds + Staged<D>::kScale + 4 * (32 + 16 * u + 4 * g));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool there = t0 + 16 * u + 4 * g + i < p.len;
      ks[u][i] = there ? kk[i] * a.c : -1.0f;  // scales are not negative
      vs[u][i] = there ? vv[i] : 0.0f;
      vtop = fmaxf(vtop, vs[u][i]);
    }
  }
  vtop = quad_max(vtop);
  const float inv = 1.0f / vtop, faded = run.vref * inv;
  run.vref = vtop;
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int i = 0; i < 4; ++i) vs[u][i] *= inv;

  union {
    v8h v;
    v2h x[4];
  } pf[NC];
  float fade[NC];
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[n][u][i] = ks[u][i] >= 0.0f ? s[n][u][i] * ks[u][i] : -INFINITY;
        top = fmaxf(top, s[n][u][i]);
      }
    const float m = fmaxf(run.m[n], quad_max(top)), alpha = __builtin_amdgcn_exp2f(run.m[n] - m);
    run.m[n] = m;
    float sum = 0.0f;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float e[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        e[i] = __builtin_amdgcn_exp2f(s[n][u][i] - m);
        sum += e[i];
        e[i] *= vs[u][i];
      }
      pf[n].x[2 * u] = v2h{(_Float16)e[0], (_Float16)e[1]};
      pf[n].x[2 * u + 1] = v2h{(_Float16)e[2], (_Float16)e[3]};
    }
    run.l[n] = run.l[n] * alpha + sum;
    fade[n] = alpha * faded;
  }
  // lane j of a 16-lane group gives the address of row j / 2, half j % 2 of an 8 x 16 block and gets column j:
  // rows 0..3 are keys 4 g + 0..3, rows 4..7 keys 16 + 4 g + 0..3
  const int j = c16 >> 1, row = (j < 4 ? 0 : 12) + 4 * g + j;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    const v2i y = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
        (__attribute__((address_space(3))) v2i*)(lds + Staged<D>::value(row, i) + 8 * (c16 & 1)));
    const v8h vf = e4m3x8_to_f16(y[0], y[1]);
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      run.o[n][i] *= fade[n];
      run.o[n][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pf[n].v, run.o[n][i], 0, 0, 0);
    }
  }
}

// Workgroups: the prefix's parts (part, column block, head), then the sequences'
// own (part, column block, sequence, head); heads fastest, so that workgroups
// that share keys have numbers equal mod 8 (one XCD's L2) where kv_heads is a
// multiple of 8.
template <int D, int NC>
__global__ __launch_bounds__(64 * kWaves, NC == 1 ? 3 : 2) void attn_decode_kernel(DecodeArgs a) {
  constexpr int kCols = 16 * NC;
  // the waves' keys and values; behind the last step their sums
  constexpr int kWaveBytes = Staged<D>::kBytes > 16 * (D + 4) * 4 ? Staged<D>::kBytes : 16 * (D + 4) * 4;
  __shared__ __attribute__((aligned(16))) uint8_t lds[kWaves][kWaveBytes];
  __shared__ float lds_m[kWaves][kCols], lds_l[kWaves][kCols];
  const int lane = threadIdx.x & 63, g = lane >> 4, c16 = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  int item = blockIdx.x;
  const int n_prefix = a.prefix_parts * a.prefix_blocks * a.kv_heads;
  const bool shared = item < n_prefix;
  if (!shared) item -= n_prefix;
  Part p;
  p.kvh = item % a.kv_heads;
  item /= a.kv_heads;
  int b = 0, slot;
  if (!shared) {
    b = item % a.B;
    item /= a.B;
  }
  const int blocks = shared ? a.prefix_blocks : a.own_blocks;
  const int col0 = item % blocks * kCols, part = item / blocks;
  const int cols = min(kCols, (shared ? a.B * a.group : a.group) - col0);
  if (shared) {
    p.pages = a.prefix_pages;
    p.width = ((a.prefix_len - 1) >> a.page_shift) + 1;
    p.len = a.prefix_len;
    slot = part;
  } else {
    p.pages = a.pages + (int64_t)b * a.width;
    p.width = a.width;
    slot = a.prefix_parts + part;
  }
  const int64_t begin = (int64_t)part * a.part_keys;
  if (begin >= min((int64_t)p.width << a.page_shift, (int64_t)kMostKeys) && part > 0) return;  // as below, whatever the length
  // the first step's pages are on their way while the length is
  Pages first = {};
  if (p.width > 0) first = pages_of(a, p, (int)begin + wave * kKeys);
  bool bad_len = false;
  if (!shared) {
    p.len = a.lens[b];
    const int64_t most = min((int64_t)a.width << a.page_shift, (int64_t)kMostKeys);
    bad_len = p.len < 0 || p.len > most;
    p.len = p.len < 0 ? 0 : (int)min((int64_t)p.len, most);
  }
  const bool last_part = part == (shared ? a.prefix_parts : a.own_parts) - 1;
  if (bad_len && a.status && part == 0 && threadIdx.x == 0) atomicOr(a.status, MOE_DEV_BAD_LENGTH);
  if (begin >= p.len && part > 0) return;  // the join looks at lens, too
  p.begin = (int)begin;
  p.end = last_part ? p.len : (int)min((int64_t)p.len, begin + a.part_keys);

  // column n of block col0: query head (col % G) of the group, of sequence col / G in the prefix
  const auto split = [&](int col, int& seq, int& head) {
    seq = shared ? (col0 + col) / a.group : b;
    head = p.kvh * a.group + (shared ? col0 + col - seq * a.group : col0 + col);
  };
  Running<D, NC> run;
  run.vref = 0x1p-126f;  // 1 / vref stays finite
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    run.m[n] = kNoScore;
    run.l[n] = 0.0f;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) run.o[n][i] = v4f{};
  }
  int t = p.begin + wave * kKeys;
  if (t < p.end) {
    v8bf qf[NC][D / 32];
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      int seq, head;
      split(min(16 * n + c16, cols - 1), seq, head);
      const uint16_t* qrow = a.q + seq * a.q_stride + head * D + 16 * g;
#pragma unroll
      for (int i = 0; i < D / 64; ++i) {
        qf[n][2 * i] = *reinterpret_cast<const v8bf*>(qrow + 64 * i);
        qf[n][2 * i + 1] = *reinterpret_cast<const v8bf*>(qrow + 64 * i + 8);
      }
    }
    bool bad = false;
    Tile<D> x;
    Pages ahead = first;
    const auto load = [&](int at) __attribute__((always_inline)) {
      if (shared || a.own_blocks > 1)
        load_tile<D, false>(a, p, at, ahead, bad, x);
      else
        load_tile<D, true>(a, p, at, ahead, bad, x);
      ahead = pages_of(a, p, at + kStride);
    };
    load(t);
    for (; t < p.end; t += kStride)
      use_tile<D, NC>(a, p, t, x, qf, lds[wave], run, [&]() __attribute__((always_inline)) {
        if (t + kStride < p.end) load(t + kStride);
      });
    if (bad && a.status && lane == 0) atomicOr(a.status, MOE_DEV_BAD_PAGE);
  }

  // the waves' sums joined, one block of 16 columns at a time
  const bool whole = a.prefix_parts + a.own_parts == 1;
  const auto sums = [&](int w, int col) { return reinterpret_cast<float*>(lds[w]) + col * (D + 4); };
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    float l = run.l[n];
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (g == 0) {
      lds_m[wave][16 * n + c16] = run.m[n];
      lds_l[wave][16 * n + c16] = l;
    }
    __syncthreads();  // no wave needs its keys and values, or the sums of the block before, any more
#pragma unroll
    for (int i = 0; i < D / 16; ++i) *reinterpret_cast<v4f*>(sums(wave, c16) + 16 * i + 4 * g) = run.o[n][i] * run.vref;
    __syncthreads();
    const int here = min(16, cols - 16 * n);
    for (int at = threadIdx.x; at < here * (D / 4); at += 64 * kWaves) {
      const int col = at / (D / 4), d = at % (D / 4) * 4;
      float m = kNoScore;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) m = fmaxf(m, lds_m[w][16 * n + col]);
      float sum = 0.0f;
      v4f o = {};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f(lds_m[w][16 * n + col] - m);
        sum += lds_l[w][16 * n + col] * f;
        o += *reinterpret_cast<const v4f*>(sums(w, col) + d) * f;
      }
      int seq, head;
      split(16 * n + col, seq, head);
      const int64_t r = (int64_t)seq * (a.kv_heads * a.group) + head;
      if (whole) {
        const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
        *reinterpret_cast<uint2*>(a.out + r * D + d) =
            make_uint2(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv));
      } else {
        const int64_t at_part = r * (a.prefix_parts + a.own_parts) + slot;
        *reinterpret_cast<v4f*>(a.part_o + at_part * D + d) = o;
        if (d == 0) *reinterpret_cast<float2*>(a.part_ml + at_part * 2) = make_float2(m, sum);
      }
    }
  }
}

// One workgroup per output row: its parts' sums, weighed by their maxima.  Eight
// (D = 128) or sixteen parts at a time, 16 bytes a lane.
template <int D>
__global__ __launch_bounds__(256) void attn_join_kernel(DecodeArgs a) {
  constexpr int kLanes = D / 4, kAtOnce = 256 / kLanes;
  __shared__ __attribute__((aligned(16))) float lds_o[kAtOnce][D];
  __shared__ float lds_l[kAtOnce];
  const int64_t r = blockIdx.x;
  const int slots = a.prefix_parts + a.own_parts;
  const int b = (int)(r / (a.kv_heads * a.group));
  const int64_t len = min((int64_t)min(max(a.lens[b], 0), kMostKeys), (int64_t)a.width << a.page_shift);
  // parts that ran: all of the prefix's, and those of the sequence that begin before its end (the first always)
  const int used = a.prefix_parts +
                   (int)min((int64_t)a.own_parts, max((int64_t)1, (len + a.part_keys - 1) / a.part_keys));
  const float2* ml = reinterpret_cast<const float2*>(a.part_ml) + r * slots;
  float m = kNoScore;
  for (int s = threadIdx.x & 63; s < used; s += 64) m = fmaxf(m, ml[s].x);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
  const int sub = threadIdx.x % kLanes, first = threadIdx.x / kLanes;
  v4f o = {};
  float l = 0.0f;
#pragma unroll 4
  for (int s = first; s < used; s += kAtOnce) {
    const float2 x = ml[s];
    const float f = __builtin_amdgcn_exp2f(x.x - m);
    l += x.y * f;
    o += *reinterpret_cast<const v4f*>(a.part_o + (r * slots + s) * D + 4 * sub) * f;
  }
  *reinterpret_cast<v4f*>(&lds_o[first][4 * sub]) = o;
  if (sub == 0) lds_l[first] = l;
  __syncthreads();
  if (first > 0) return;
#pragma unroll
  for (int w = 1; w < kAtOnce; ++w) {
    o += *reinterpret_cast<const v4f*>(&lds_o[w][4 * sub]);
    l += lds_l[w];
  }
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
  *reinterpret_cast<uint2*>(a.out + r * D + 4 * sub) =
      make_uint2(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv));
}

struct DecodePlan {
  int part_keys, prefix_parts, own_parts, prefix_blocks, own_blocks, col_blocks;
  int64_t slots_of_rows;  // B * q_heads * slots where there is more than one slot
};

DecodePlan plan_decode(const moe_attn_dims_t& d, int32_t B, int32_t max_len, int32_t prefix_len) {
  DecodePlan p{};
  const int group = d.q_heads / d.kv_heads;
  p.col_blocks = group > 16 || (prefix_len > 0 && (int64_t)B * group > 16) ? 2 : 1;
  p.own_blocks = (group + 16 * p.col_blocks - 1) / (16 * p.col_blocks);
  p.prefix_blocks = (int)(((int64_t)B * group + 16 * p.col_blocks - 1) / (16 * p.col_blocks));
  const int64_t keys = ((int64_t)B * p.own_blocks * max_len + (int64_t)p.prefix_blocks * prefix_len) * d.kv_heads;
  const int64_t even = (keys + 511) / 512;
  p.part_keys = (int)std::min<int64_t>(1024, std::max<int64_t>(256, (even + kStride - 1) / kStride * kStride));
  p.own_parts = std::max(1, (int)(((int64_t)max_len + p.part_keys - 1) / p.part_keys));
  p.prefix_parts = (int)(((int64_t)prefix_len + p.part_keys - 1) / p.part_keys);
  const int slots = p.own_parts + p.prefix_parts;
  p.slots_of_rows = slots > 1 ? (int64_t)B * d.q_heads * slots : 0;
  return p;
}

size_t part_bytes(const DecodePlan& p, int width) {
  return ((size_t)p.slots_of_rows * width * sizeof(float) + 255) & ~(size_t)255;
}

template <int D>
moe_status_t launch_decode(const DecodeArgs& a, const DecodePlan& p, hipStream_t stream) {
  const int64_t items = ((int64_t)p.prefix_parts * p.prefix_blocks + (int64_t)p.own_parts * p.own_blocks * a.B) * a.kv_heads;
  const int64_t rows = (int64_t)a.B * a.kv_heads * a.group;
  if (items * 64 * kWaves >= (int64_t)1 << 32 || rows * 256 >= (int64_t)1 << 32)
    return fail(MOE_ERR_UNSUPPORTED_SHAPE, "moe_attn_decode: %lld parts", (long long)items);
  if (p.col_blocks == 1)
    MOE_LAUNCH("attn_decode", (attn_decode_kernel<D, 1>), dim3((unsigned)items), dim3(64 * kWaves), 0, stream, a);
  else
    MOE_LAUNCH("attn_decode", (attn_decode_kernel<D, 2>), dim3((unsigned)items), dim3(64 * kWaves), 0, stream, a);
  if (p.slots_of_rows)
    MOE_LAUNCH("attn_join", attn_join_kernel<D>, dim3((unsigned)rows), dim3(256), 0, stream, a);
  return check_launch("moe_attn_decode");
}

}  // namespace

}  // namespace moe

using namespace moe;

extern "C" size_t moe_attn_decode_workspace(moe_attn_dims_t d, int32_t B, int32_t max_len, int32_t prefix_len) {
  if (check_attn_dims(d, "moe_attn_decode_workspace") != MOE_OK || B < 1 || B > 65535 || max_len < 0 || prefix_len < 0 ||
      max_len > kMostKeys || prefix_len > kMostKeys)
    return 0;
  const DecodePlan p = plan_decode(d, B, max_len, prefix_len);
  return part_bytes(p, d.head_dim) + part_bytes(p, 2);
}

extern "C" moe_status_t moe_attn_decode(moe_attn_dims_t d, int32_t B, const uint16_t* q, int64_t q_stride,
                                        moe_kv_cache_t cache, const int32_t* page_table, int32_t table_width,
                                        const int32_t* lens, int32_t max_len, const int32_t* prefix_pages,
                                        int32_t prefix_len, float scale, uint16_t* out, int32_t* dev_status, void* ws,
                                        size_t ws_bytes, hipStream_t stream) {
  moe_status_t st = check_attn_dims(d, "moe_attn_decode");
  if (st != MOE_OK) return st;
  if ((st = check_cache(cache, "moe_attn_decode")) != MOE_OK) return st;
  if (B < 0 || B > 65535 || table_width < 0 || max_len < 0 || prefix_len < 0 || max_len > kMostKeys ||
      prefix_len > kMostKeys)
    return fail(MOE_ERR_INVALID_ARG,
                "moe_attn_decode: B=%d (at most 65535) table_width=%d max_len=%d prefix_len=%d (at most 2^30)", B,
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
  const DecodePlan p = plan_decode(d, B, max_len, prefix_len);
  uint8_t* base = static_cast<uint8_t*>(ws);
  float* part_o = p.slots_of_rows ? reinterpret_cast<float*>(base) : nullptr;
  float* part_ml = p.slots_of_rows ? reinterpret_cast<float*>(base + part_bytes(p, d.head_dim)) : nullptr;
  const DecodeArgs a{q, q_stride, cache, page_table, lens, prefix_pages, out, part_o, part_ml, dev_status, B, table_width,
                     prefix_len, d.kv_heads, d.q_heads / d.kv_heads, __builtin_ctz((unsigned)cache.page_size),
                     p.part_keys, p.prefix_parts, p.own_parts, p.prefix_blocks, p.own_blocks, scale * kLog2e};
  return d.head_dim == 64 ? launch_decode<64>(a, p, stream) : launch_decode<128>(a, p, stream);
}
