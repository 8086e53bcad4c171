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
//   O^T = V^T P^T (bf16) values' codes go through LDS and come back transposed
//                 (ds_read_b64_tr_b8) in the order of keys that the scores have
// Scales stay fp32: a key's multiplies its score, a value's its numerator.  The
// products of these are split into two bf16, a rounded one and what it leaves (16
// bits of mantissa, the exponents of fp32), each multiplied: the matrix cores have
// the time, and the result is exact but for its own rounding (1.7e-3 of its norm;
// with one bf16 2.4e-3).
//
// Bound by memory: head_dim + 4 bytes per key, value and head against 4 * G *
// head_dim flops.  64 sequences of up to 8192 keys: 77 us, 5.2 TB/s (a kernel that
// only loads the same takes as long), and 81 with the join; one of 65536: 25 us, 5.5
// TB/s, and 34 until the join has ended.  On a prefix, where a key serves 16 NCP
// columns, by latencies: 48 sequences behind 8191 shared keys 26 us, of which 15 are
// eight steps of about 330 instructions beside 48 MFMAs, two waves to a SIMD, and the
// rest is finding the piece, the first loads and joining the waves' sums (vector
// instructions take 26 % of the SIMDs' cycles, the matrix cores 13 %).
//
// A head's work is a line of steps of 128 keys (32 for each wave of a
// workgroup): the prefix's for every block of columns, then the sequences' one
// behind the other.  The workgroups that the card holds at once take equal pieces
// of the heads' lines, so that one long context and a ragged batch both fill it
// evenly; where a piece or a sequence ends, a segment ends, whose sums a second
// launch joins.  Short contexts take one workgroup a sequence and head, which walks
// the prefix for itself, and no second launch.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "attention.h"

namespace moe {

namespace {

struct DecodeArgs {
  const uint16_t* q;
  int64_t q_stride;
  moe_kv_cache_t cache;
  const int32_t *pages, *lens, *prefix_pages;
  uint16_t* out;
  float* seg_o;     // [segments][columns][D]: a segment's sums, not divided
  float2* seg_ml;   // [segments][columns]: its running maxima and sums
  uint32_t* starts;  // [B + 1]: a sequence's first step in a head's line; [B]: the line's length
  int32_t* status;
  int B, width, prefix_len, kv_heads, group, page_shift;
  int prefix_blocks, own_blocks;  // column blocks of all sequences' and of one's queries
  int pieces;                     // that a head's line is cut into
  float c;                        // scale * log2(e)
};

constexpr int kKeys = 32;  // keys per step of a wave
constexpr int kWaves = 4;
constexpr int kStride = kKeys * kWaves;  // keys per step of a workgroup
constexpr int kMostKeys = 1 << 30;  // of a sequence: key indices and the steps behind them stay in 32 bits

// The running softmax of NC blocks of 16 queries; a lane's query is column
// lane % 16 of each block.
template <int D, int NC>
struct Running {
  v4f o[NC][D / 16];   // O^T: rows 16 i + 4 (lane / 16) + 0..3
  float m[NC], l[NC];  // l: this lane's keys only, summed over the lane groups at the end
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
// Each half of the wave looks at one: a value of the lanes, which becomes a scalar
// where the loads behind it need it.  (A load of one address for all lanes is made
// a scalar at once, behind a wait for every load in front of it, the step's keys
// and values among them.)
__device__ __forceinline__ int pages_of(const DecodeArgs& a, const Part& p, int t) {
  const int lane = threadIdx.x, half = (lane & 32) >> 1;
  return p.pages[(uint32_t)min((t + half) >> a.page_shift, p.width - 1)];
}

// A wave's part of LDS: keys, values (rows of D codes), scales.  Rows are 16 bytes
// longer than their codes, so that 16 of them at one chunk of 16 bytes lie in
// different banks, and all places of a lane are one register and constants.
// Values stand in the order in which a transposed read takes them: keys 4 g + 0..3
// and 16 + 4 g + 0..3 as rows 8 g + 0..7.
template <int D>
struct Staged {
  static constexpr int kPitch = D + 16, kV = kKeys * kPitch, kScale = 2 * kV, kBytes = kScale + 64 * 4;
  static __device__ __forceinline__ int key(int row, int c) { return row * kPitch + 16 * c; }
  static __device__ __forceinline__ int value(int row, int c) {
    return kV + (((row & 12) << 1) | ((row & 16) >> 2) | (row & 3)) * kPitch + 16 * c;
  }
};

// Loads keys [t0, t0 + 32), t0 < len.  Keys behind the end repeat the last, or
// the first half where the second holds none.  kOnce: nothing else reads them in
// this launch, so they need no place in the caches (64 ragged contexts: 90 us
// without, 78 with, whole rows per load in both).
template <int D, bool kOnce>
__device__ __forceinline__ void load_tile(const DecodeArgs& a, const Part& p, const float* scales, int t0, int pages,
                                          bool& bad, Tile<D>& x) {
  constexpr int kChunks = D / 16;
  const int lane = threadIdx.x & 63, mask = a.cache.page_size - 1, last = p.len - 1;
  const bool two = t0 + 16 <= last;
  const int id0 = __builtin_amdgcn_readlane(pages, 0), id1 = two ? __builtin_amdgcn_readlane(pages, 32) : id0;
  const bool wrong0 = id0 < 0 || id0 >= a.cache.n_pages, wrong1 = id1 < 0 || id1 >= a.cache.n_pages;
  bad |= wrong0 | wrong1;
  // the first key of each half, counted in rows of the cache
  const int64_t row0 = (((int64_t)(wrong0 ? 0 : id0) * a.kv_heads + p.kvh) << a.page_shift) + (t0 & mask);
  const int64_t row1 = two ? (((int64_t)(wrong1 ? 0 : id1) * a.kv_heads + p.kvh) << a.page_shift) + ((t0 + 16) & mask) : row0;
  const int left = last - t0, left1 = two ? left - 16 : left;  // rows behind these repeat them
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    // scalar bases and 32-bit offsets
    const bool second = i >= D / 64;
    const int row = 64 / kChunks * (i % (D / 64)) + lane / kChunks;
    const uint32_t from = min(row, second ? left1 : left) * D + lane % kChunks * 16;
    const int64_t base = (second ? row1 : row0) * D;
    const u32x4_stream* k = reinterpret_cast<const u32x4_stream*>(a.cache.k + base + from);
    const u32x4_stream* v = reinterpret_cast<const u32x4_stream*>(a.cache.v + base + from);
    x.k[i] = kOnce ? __builtin_nontemporal_load(k) : *k;
    x.v[i] = kOnce ? __builtin_nontemporal_load(v) : *v;
  }
  const int row = lane & 15;
  x.scale = scales[(lane & 16 ? row1 : row0) + min(row, lane & 16 ? left1 : left)];
}

__device__ __forceinline__ float most(v4f a, v4f b) {
  return fmaxf(fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3])), fmaxf(fmaxf(b[0], b[1]), fmaxf(b[2], b[3])));
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
  *reinterpret_cast<float*>(lds + Staged<D>::kScale + 4 * lane) = lane < 32 ? x.scale * a.c : x.scale;
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
      for (int n = 0; n < NC; ++n) s[n][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lo, qf[n][2 * i], s[n][u], 0, 0, 0);
#pragma unroll
      for (int n = 0; n < NC; ++n)
        s[n][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi, qf[n][2 * i + 1], s[n][u], 0, 0, 0);
    }
  }
  v4f ks[2], vs[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    ks[u] = *reinterpret_cast<const v4f*>(lds + Staged<D>::kScale + 4 * (16 * u + 4 * g));
    vs[u] = *reinterpret_cast<const v4f*>(lds + Staged<D>::kScale + 4 * (32 + 16 * u + 4 * g));
  }
  if (t0 + kKeys > p.len) {  // a slot behind the end may hold any bits
    asm volatile("");        // one step of many: no selects in the others
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool there = t0 + 16 * u + 4 * g + i < p.len;
        ks[u][i] = there ? ks[u][i] : 1.0f;
        vs[u][i] = there ? vs[u][i] : 0.0f;
#pragma unroll
        for (int n = 0; n < NC; ++n) s[n][u][i] = there ? s[n][u][i] : -INFINITY;
      }
  }
  // the logarithms of the numerators under the maxima so far
  v4f e[NC][2];
  bool grows = false;
#pragma unroll
  for (int n = 0; n < NC; ++n) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) e[n][u][i] = fmaf(s[n][u][i], ks[u][i], -run.m[n]);
    grows |= most(e[n][0], e[n][1]) > 8.0f;
  }
  // Rescaled only when a maximum grows by more than 2^8: numerators up to 2^8 are as exact.  The lanes of a query have
  // one maximum, so that only then do they have to agree on another.
  if (__any(grows)) {
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      v4f x[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) x[u] = s[n][u] * ks[u];
      const float m = fmaxf(run.m[n], quad_max(most(x[0], x[1]))), alpha = __builtin_amdgcn_exp2f(run.m[n] - m);
      run.m[n] = m;
      run.l[n] *= alpha;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) run.o[n][i] *= alpha;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) e[n][u][i] = fmaf(s[n][u][i], ks[u][i], -m);
    }
  }
  union {
    v8bf v;
    uint32_t x[4];
  } hi[NC], lo[NC];
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    float sum = 0.0f;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w[i] = __builtin_amdgcn_exp2f(e[n][u][i]);
        sum += w[i];
        w[i] *= vs[u][i];
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t x = pack_bf16(w[2 * i], w[2 * i + 1]);
        hi[n].x[2 * u + i] = x;
        lo[n].x[2 * u + i] = pack_bf16(w[2 * i] - __uint_as_float(x << 16), w[2 * i + 1] - __uint_as_float(x & 0xffff0000u));
      }
    }
    run.l[n] += sum;
  }
  // lane j of a 16-lane group gives the address of row j / 2, half j % 2 of an 8 x 16 block and gets column j
  const uint8_t* at = lds + Staged<D>::kV + (8 * g + (c16 >> 1)) * Staged<D>::kPitch + 8 * (c16 & 1);
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    const v2i y = __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) v2i*)(at + 16 * i));
    const v8bf vf = e4m3x8_to_bf16(y[0], y[1]);
#pragma unroll
    for (int n = 0; n < NC; ++n) run.o[n][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, hi[n].v, run.o[n][i], 0, 0, 0);
#pragma unroll
    for (int n = 0; n < NC; ++n) run.o[n][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, lo[n].v, run.o[n][i], 0, 0, 0);
  }
}

// Steps of a run of keys.
__host__ __device__ __forceinline__ int steps_of(int keys) { return (keys + kStride - 1) / kStride; }

// A head's line of steps, and its pieces: prefix_blocks times the prefix's steps,
// own_blocks times all sequences'.  (The host checks that it has less than 2^31
// steps.)  A pair is one of its runs of keys for one block of columns: the
// prefix's blocks, then (block, sequence).  Pieces and pairs end one at a time, so
// that segments are numbered by the sum of their piece's and their pair's number.
struct Line {
  uint32_t prefix_steps, prefix_total, own_total;
  uint32_t base, more;  // a piece has base steps, the first `more` have one more
  int64_t segments;     // of a head, at most
  __device__ __forceinline__ Line(const DecodeArgs& a, uint32_t own) {
    prefix_steps = steps_of(a.prefix_len);
    prefix_total = prefix_steps * a.prefix_blocks;
    own_total = own;
    const uint32_t all = prefix_total + own * a.own_blocks;
    base = all / (uint32_t)a.pieces;
    more = all - base * a.pieces;
    segments = (int64_t)a.pieces + a.prefix_blocks + (int64_t)a.own_blocks * a.B;
  }
  __device__ __forceinline__ uint32_t begin(uint32_t piece) const { return piece * base + min(piece, more); }
  __device__ __forceinline__ uint32_t piece_of(uint32_t step) const {
    const uint32_t longer = more * (base + 1);
    return step < longer ? step / (base + 1) : more + (step - longer) / max(base, 1u);
  }
};

// A sequence's own keys, cut to its page table row, and its steps.
__device__ __forceinline__ int keys_of(const DecodeArgs& a, int b, bool& bad) {
  const int len = a.lens[b];
  const int64_t most = min((int64_t)a.width << a.page_shift, (int64_t)kMostKeys);
  bad = len < 0 || len > most;
  return len < 0 ? 0 : (int)min((int64_t)len, most);
}

// 64 sequences' steps, a lane each, and their sum up to each.
struct Chunk {
  int base = -1, len, n, incl;
  __device__ __forceinline__ void load(const DecodeArgs& a, int from, bool report) {
    if (from == base) return;
    base = from;
    const int b = from + (threadIdx.x & 63);
    bool bad = false;
    len = b < a.B ? keys_of(a, b, bad) : 0;
    if (report && bad && a.status) atomicOr(a.status, MOE_DEV_BAD_LENGTH);
    n = steps_of(len);
    incl = wave_scan(n);
  }
};

// kWhole: a workgroup takes all keys of one (sequence, head, block of columns),
// the prefix's first, and writes its output; otherwise a piece of the line.
// NCP, NCO: blocks of 16 columns on the prefix's keys and on a sequence's own.
template <int D, int NCP, int NCO, bool kWhole>
__global__ __launch_bounds__(64 * kWaves, 2) void attn_decode_kernel(DecodeArgs a) {
  constexpr int kCols = 16 * (NCP > NCO ? NCP : NCO);
  // the waves' keys and values; behind the last step their sums
  constexpr int kWaveBytes = Staged<D>::kBytes > 16 * (D + 4) * 4 ? Staged<D>::kBytes : 16 * (D + 4) * 4;
  __shared__ __attribute__((aligned(16))) uint8_t lds[kWaves][kWaveBytes];
  __shared__ float lds_m[kWaves][kCols], lds_l[kWaves][kCols];
  const int lane = threadIdx.x & 63, g = lane >> 4, c16 = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  // keys' scales for the lanes that load those, values' for the others
  const float* scales = lane < 32 ? a.cache.k_scale : a.cache.v_scale;
  using Front = std::integral_constant<int, NCP>;
  using Own = std::integral_constant<int, NCO>;
  Part p;
  const auto prefix_part = [&](int begin, int end) __attribute__((always_inline)) {
    return Part{a.prefix_pages, ((a.prefix_len - 1) >> a.page_shift) + 1, a.prefix_len, begin, end, p.kvh};
  };
  bool shared = false;
  int b = 0, col0 = 0, cols = 0;
  int64_t segment = 0;
  // The segment's keys by p, the sums to `segment` or (kWhole) the output.  kWhole: the prefix's keys in front of them.
  const auto run_segment = [&](auto blocks, int first) __attribute__((always_inline)) {
    constexpr int NC = decltype(blocks)::value;
    // column n of block col0: query head (col % G) of the group, of sequence col / G in the prefix
    const auto split = [&](int col, int& seq, int& head) {
      seq = shared ? (col0 + col) / a.group : b;
      head = p.kvh * a.group + (shared ? col0 + col - seq * a.group : col0 + col);
    };
    Running<D, NC> run;
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      run.m[n] = kNoScore;
      run.l[n] = 0.0f;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) run.o[n][i] = v4f{};
    }
    if (kWhole || p.begin + wave * kKeys < p.end) {
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
      const auto walk = [&](const Part& p, bool again, int ahead) __attribute__((always_inline)) {
        int t = p.begin + wave * kKeys;
        if (t >= p.end) return;
        Tile<D> x;
        const auto load = [&](int at) __attribute__((always_inline)) {
          if (again)
            load_tile<D, false>(a, p, scales, at, ahead, bad, x);
          else
            load_tile<D, true>(a, p, scales, at, ahead, bad, x);
          ahead = pages_of(a, p, at + kStride);
        };
        load(t);
        for (; t < p.end; t += kStride)
          use_tile<D, NC>(a, p, t, x, qf, lds[wave], run, [&]() __attribute__((always_inline)) {
            if (t + kStride < p.end) load(t + kStride);
          });
      };
      if (kWhole && a.prefix_len > 0) {
        const Part front = prefix_part(0, a.prefix_len);
        walk(front, true, pages_of(a, front, wave * kKeys));
      }
      walk(p, shared || a.own_blocks > 1, first);
      if (bad && a.status && lane == 0) atomicOr(a.status, MOE_DEV_BAD_PAGE);
    }

    // the waves' sums joined, one block of 16 columns at a time
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
      for (int i = 0; i < D / 16; ++i) *reinterpret_cast<v4f*>(sums(wave, c16) + 16 * i + 4 * g) = run.o[n][i];
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
        if (kWhole) {
          int seq, head;
          split(16 * n + col, seq, head);
          const int64_t r = (int64_t)seq * (a.kv_heads * a.group) + head;
          const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
          *reinterpret_cast<uint2*>(a.out + r * D + d) =
              make_uint2(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv));
        } else {
          const int64_t place = segment * kCols + 16 * n + col;
          *reinterpret_cast<v4f*>(a.seg_o + place * D + d) = o;
          if (d == 0) a.seg_ml[place] = make_float2(m, sum);
        }
      }
    }
  };

  if (kWhole) {
    int item = blockIdx.x;
    p.kvh = item % a.kv_heads;
    item /= a.kv_heads;
    b = item % a.B;
    col0 = item / a.B * 16 * NCO;
    cols = min(16 * NCO, a.group - col0);
    p.pages = a.pages + (int64_t)b * a.width;
    p.width = a.width;
    // the first step's pages are on their way while the length is
    int first = 0;
    if (a.width > 0) first = pages_of(a, p, wave * kKeys);
    bool bad;
    p.len = keys_of(a, b, bad);
    if (bad && a.status && threadIdx.x == 0) atomicOr(a.status, MOE_DEV_BAD_LENGTH);
    p.begin = 0;
    p.end = p.len;
    run_segment(Own{}, first);
    return;
  }

  // Heads fastest: the heads of a page are read at one time, and workgroups that share keys (the prefix's blocks of
  // columns) have numbers equal mod 8 (one XCD's L2) where kv_heads is a multiple of 8.
  p.kvh = blockIdx.x % (uint32_t)a.kv_heads;
  const uint32_t piece = blockIdx.x / (uint32_t)a.kv_heads;
  // The first wave finds the segments of this workgroup's piece, one at a time; the others take what it found, so that
  // all leave together whatever the lengths in memory do.
  __shared__ struct {
    int more, shared, col0, cols, b, len, begin, end;
    uint32_t pair;
  } found;
  Chunk chunk;
  uint32_t own = 0;
  if (wave == 0) {
    // the line's length; the first workgroup leaves every sequence's place in it to the join
    for (int from = 0; from < a.B; from += 64) {
      chunk.load(a, from, blockIdx.x == 0);
      if (blockIdx.x == 0 && from + lane < a.B) a.starts[from + lane] = own + chunk.incl - chunk.n;
      own += __builtin_amdgcn_readlane(chunk.incl, 63);
    }
    if (blockIdx.x == 0 && lane == 0) a.starts[a.B] = own;
  }
  const Line line(a, own);
  const uint32_t end = line.begin(piece + 1);
  uint32_t at = line.begin(piece), block_at = ~0u, before = 0;  // chunk is of this block's sequences, steps in front of it
  while (true) {
    if (wave == 0) {
      uint32_t pair = 0, skip = 0, steps = 0;  // the pair, its steps in front of `at`, and those that are left
      uint32_t block = 0;
      int seq = 0, len = 0;
      const bool front = at < line.prefix_total;
      if (at >= end) {
      } else if (front) {
        pair = block = at / line.prefix_steps;
        skip = at - block * line.prefix_steps;
        steps = line.prefix_steps - skip;
        len = a.prefix_len;
      } else {
        const uint32_t own_at = at - line.prefix_total;
        block = a.own_blocks == 1 ? 0 : own_at / line.own_total;
        const uint32_t in_block = own_at - block * line.own_total;
        int from = block == block_at ? chunk.base : 0;
        if (block != block_at) before = 0;
        block_at = block;
        for (; from < a.B; from += 64) {
          chunk.load(a, from, false);
          const uint64_t past = __ballot(before + chunk.incl > in_block);
          if (past) {
            const int w = __ffsll((unsigned long long)past) - 1, n = __builtin_amdgcn_readlane(chunk.n, w);
            seq = from + w;
            skip = in_block - (before + __builtin_amdgcn_readlane(chunk.incl, w) - n);
            steps = n - skip;
            len = __builtin_amdgcn_readlane(chunk.len, w);
            break;
          }
          before += __builtin_amdgcn_readlane(chunk.incl, 63);
        }
        pair = a.prefix_blocks + block * a.B + seq;
      }
      const uint32_t taken = min(steps, end - at);
      if (lane == 0) {
        found.more = taken > 0;
        found.shared = front;
        const int width = 16 * (front ? NCP : NCO);
        found.col0 = block * width;
        found.cols = min(width, (front ? a.B * a.group : a.group) - (int)block * width);
        found.b = seq;
        found.len = len;
        found.begin = (int)(skip * kStride);
        found.end = min(len, (int)((skip + taken) * kStride));
        found.pair = pair;
      }
      at += taken;
    }
    __syncthreads();  // (and the sums' places may take the next segment's keys)
    if (!found.more) return;
    shared = __builtin_amdgcn_readfirstlane(found.shared);
    col0 = __builtin_amdgcn_readfirstlane(found.col0);
    cols = __builtin_amdgcn_readfirstlane(found.cols);
    b = __builtin_amdgcn_readfirstlane(found.b);
    p.len = __builtin_amdgcn_readfirstlane(found.len);
    p.begin = __builtin_amdgcn_readfirstlane(found.begin);
    p.end = __builtin_amdgcn_readfirstlane(found.end);
    segment = p.kvh * line.segments + piece + (uint32_t)__builtin_amdgcn_readfirstlane(found.pair);
    if (shared) {
      p = prefix_part(p.begin, p.end);
    } else {
      p.pages = a.pages + (int64_t)b * a.width;
      p.width = a.width;
    }
    const int first = pages_of(a, p, p.begin + wave * kKeys);
    if (NCP != NCO && shared)
      run_segment(Front{}, first);
    else
      run_segment(Own{}, first);
  }
}

// A row's segments, weighed by their maxima: those of the prefix's pair that has
// the row among its columns, then those of the row's own.  D / 4 lanes with 16
// bytes each take a segment; kAtOnce of them work on one row.
template <int D, int NCP, int NCO, int kAtOnce>
__global__ __launch_bounds__(256) void attn_join_kernel(DecodeArgs a) {
  constexpr int kCols = 16 * (NCP > NCO ? NCP : NCO), kPrefixCols = 16 * NCP, kOwnCols = 16 * NCO, kLanes = D / 4, kRows = 256 / (kLanes * kAtOnce);
  __shared__ __attribute__((aligned(16))) float lds_o[kAtOnce][D];
  __shared__ float lds_m[kAtOnce], lds_l[kAtOnce];
  const int sub = threadIdx.x % kLanes, nth = threadIdx.x / kLanes % kAtOnce;
  const int heads = a.kv_heads * a.group;
  const int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / (kLanes * kAtOnce);
  if (r >= (int64_t)a.B * heads) return;  // (kAtOnce > 1: one row a workgroup)
  const int b = (int)((uint32_t)r / (uint32_t)heads), head = (int)(r - (int64_t)b * heads);
  const int kvh = head / a.group, col = head - kvh * a.group;
  const uint32_t start = a.starts[b], steps = a.starts[b + 1] - start;
  const Line line(a, a.starts[a.B]);
  float m = kNoScore, l = 0.0f;
  v4f o = {};
  const auto take = [&](uint32_t pair, uint32_t first, uint32_t last, int column) __attribute__((always_inline)) {
    const uint32_t w0 = line.piece_of(first), w1 = line.piece_of(last);
    const int64_t place0 = (kvh * line.segments + pair) * kCols + column;
#pragma unroll 4
    for (uint32_t w = w0 + nth; w <= w1; w += kAtOnce) {
      const int64_t place = place0 + (int64_t)w * kCols;
      const float2 ml = a.seg_ml[place];
      const v4f x = *reinterpret_cast<const v4f*>(a.seg_o + place * D + 4 * sub);
      const float top = fmaxf(m, ml.x), f = __builtin_amdgcn_exp2f(m - top), e = __builtin_amdgcn_exp2f(ml.x - top);
      m = top;
      l = l * f + ml.y * e;
      o = o * f + x * e;
    }
  };
  if (a.prefix_len > 0) {
    const int pcol = b * a.group + col;
    const uint32_t block = pcol / kPrefixCols;
    take(block, block * line.prefix_steps, (block + 1) * line.prefix_steps - 1, pcol % kPrefixCols);
  }
  if (steps > 0) {
    const uint32_t block = col / kOwnCols, first = line.prefix_total + block * line.own_total + start;
    take(a.prefix_blocks + block * a.B + b, first, first + steps - 1, col % kOwnCols);
  }
  if (kAtOnce > 1) {
    *reinterpret_cast<v4f*>(&lds_o[nth][4 * sub]) = o;
    if (sub == 0) {
      lds_m[nth] = m;
      lds_l[nth] = l;
    }
    __syncthreads();
    if (nth > 0) return;
    float top = m;
#pragma unroll
    for (int w = 1; w < kAtOnce; ++w) top = fmaxf(top, lds_m[w]);
    const float f = __builtin_amdgcn_exp2f(m - top);
    o *= f;
    l *= f;
#pragma unroll
    for (int w = 1; w < kAtOnce; ++w) {
      const float e = __builtin_amdgcn_exp2f(lds_m[w] - top);
      o += *reinterpret_cast<const v4f*>(&lds_o[w][4 * sub]) * e;
      l += lds_l[w] * e;
    }
  }
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
  *reinterpret_cast<uint2*>(a.out + r * D + 4 * sub) =
      make_uint2(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv));
}

struct DecodePlan {
  bool whole;
  int front, own;  // blocks of 16 columns in a workgroup, on the prefix's keys and on a sequence's own
  int own_blocks, prefix_blocks, pieces;
  int64_t workgroups;
  size_t o_bytes, ml_bytes, start_bytes;
  size_t bytes() const { return o_bytes + ml_bytes + start_bytes; }
};

// What one launch, in which a workgroup walks all keys of a sequence and head, the
// prefix's for each sequence anew, saves against equal pieces and a join.
// Estimates in us, of D = 128 (D = 64 is quicker on both sides).  One launch: 0.9 a
// step, more when more than 256 workgroups share the card (a sequence's own steps,
// most of them fewer than the longest's, when more than 384).  Two: 5 us more to
// begin with, 6 with a prefix, what a sequence costs to begin and end, and the
// pieces' steps, a prefix's with twice the columns.  32 heads over 8, one launch
// against two: 1 sequence of 512 keys 6.8 against 8.2, of 1024 10.6 against 8.4; 32
// of up to 1024 11.9 against 14.6, of up to 2048 19.3 against 18.6; 48 of up to 500
// behind 120 shared ones 11.5 against 16.4, of up to 250 behind 1500 23 against 19.
// The estimates know neither the memory's rate nor how the lengths differ: 48 of 4000
// keys each 75 us in one launch (which they choose) and 76 in two, of up to 4000 40
// and 34.
double whole_gains(const DecodePlan& p, const moe_attn_dims_t& d, int32_t B, int32_t own_steps, int32_t prefix_steps) {
  const double groups = (double)p.own_blocks * B * d.kv_heads;
  const double line = 2.0 * p.prefix_blocks * prefix_steps + (double)p.own_blocks * B * own_steps;
  const double one = 3.2 + 0.9 * (own_steps * std::max(1.0, groups / 384) + prefix_steps * std::max(1.0, groups / 256));
  const double two = (prefix_steps > 0 ? 9.5 : 8.2) + 3.2 * groups / 512 + 0.9 * line * d.kv_heads / 512;
  return two - one;
}

// The columns' blocks: all that the choice between one launch and two looks at.
DecodePlan plan_blocks(const moe_attn_dims_t& d, int32_t B, int32_t prefix_len) {
  DecodePlan p{};
  const int group = d.q_heads / d.kv_heads;
  const int64_t all = (int64_t)B * group;
  p.own = group > 16 ? 2 : 1;
  // two blocks of columns a wave on the prefix (48 sequences of 4 columns each, 8191 keys: 28 us; one block 39, four, with
  // one workgroup a CU, 40)
  p.front = prefix_len > 0 && all > 16 ? 2 : p.own;
  p.own_blocks = (group + 16 * p.own - 1) / (16 * p.own);
  p.prefix_blocks = prefix_len > 0 ? (int)((all + 16 * p.front - 1) / (16 * p.front)) : 0;
  return p;
}

// Equal pieces and a join.  Everything here only grows with B, max_len and prefix_len.
DecodePlan plan_pieces(const moe_attn_dims_t& d, int32_t B, int32_t max_len, int32_t prefix_len) {
  DecodePlan p = plan_blocks(d, B, prefix_len);
  const int64_t own_pairs = (int64_t)p.own_blocks * B;
  const int64_t steps = own_pairs * steps_of(max_len) + (int64_t)p.prefix_blocks * steps_of(prefix_len);
  // Two workgroups a CU (64 ragged contexts: 77 us with 512 workgroups, 81 with 768, 84 with 1536; one context of 65536:
  // 27, 29 and 31 us, and a longer join).
  // Fewer where a row would have many segments of few steps: steps / pieces in the first launch and pieces / runs of keys
  // in the second cost about as much at this number (16 heads over 1, one context of 65536, 80 pieces 11.6 + 5.3 us, 512
  // 8.1 + 24.4; 28 over 4, two of up to 16583, 80 pieces 8.6 + 6.4, 128 9.1 + 8.2).
  const int64_t few = (int64_t)ceil(3.5 * sqrt((double)steps * (double)(p.prefix_blocks + own_pairs)));
  p.pieces = (int)std::max<int64_t>(1, std::min(std::min<int64_t>(512 / d.kv_heads, few), steps));
  p.workgroups = (int64_t)p.pieces * d.kv_heads;
  const size_t places = (size_t)d.kv_heads * (p.pieces + p.prefix_blocks + own_pairs) * 16 * std::max(p.front, p.own);
  p.o_bytes = (places * d.head_dim * sizeof(float) + 255) & ~(size_t)255;
  p.ml_bytes = (places * sizeof(float2) + 255) & ~(size_t)255;
  p.start_bytes = ((size_t)(B + 1) * sizeof(uint32_t) + 255) & ~(size_t)255;
  return p;
}

DecodePlan plan_decode(const moe_attn_dims_t& d, int32_t B, int32_t max_len, int32_t prefix_len) {
  DecodePlan p = plan_blocks(d, B, prefix_len);
  p.whole = whole_gains(p, d, B, steps_of(max_len), steps_of(prefix_len)) >= 0.0;
  if (!p.whole) return plan_pieces(d, B, max_len, prefix_len);
  p.workgroups = (int64_t)p.own_blocks * B * d.kv_heads;
  return p;
}

// What a call of these sizes or smaller ones may need.  A longer context or prefix never makes one launch the faster
// form, but for a prefix at all (the join costs more with one); a larger batch can, since its workgroups share the card.
// So the largest batch that would take two launches, with the prefix or without, decides.
size_t decode_workspace(const moe_attn_dims_t& d, int32_t B, int32_t max_len, int32_t prefix_len) {
  constexpr double kRounding = 1e-9;  // us: of estimates that are equal but for the order of their sums
  for (int32_t b = B; b > 0; --b)
    for (const int32_t prefix : {prefix_len, 0})
      if (whole_gains(plan_blocks(d, b, prefix), d, b, steps_of(max_len), steps_of(prefix)) < kRounding)
        return plan_pieces(d, b, max_len, prefix_len).bytes();
  return 0;
}

template <int D, int NCP, int NCO>
moe_status_t launch_decode(const DecodeArgs& a, const DecodePlan& p, hipStream_t stream) {
  constexpr int kAtOnce = 256 / (D / 4);
  const int64_t rows = (int64_t)a.B * a.kv_heads * a.group;
  if (std::max(p.workgroups, rows) * 64 * kWaves >= (int64_t)1 << 32)
    return fail(MOE_ERR_UNSUPPORTED_SHAPE, "moe_attn_decode: %lld rows", (long long)rows);
  const dim3 grid((unsigned)p.workgroups);
  if (p.whole) {
    MOE_LAUNCH("attn_decode", (attn_decode_kernel<D, NCO, NCO, true>), grid, dim3(64 * kWaves), 0, stream, a);
    return check_launch("moe_attn_decode");
  }
  MOE_LAUNCH("attn_decode", (attn_decode_kernel<D, NCP, NCO, false>), grid, dim3(64 * kWaves), 0, stream, a);
  // A row has about as many segments as its pairs have pieces: a workgroup a row for many, lanes of their own for few.
  if (p.pieces >= 4 * (p.prefix_blocks + p.own_blocks * a.B))
    MOE_LAUNCH("attn_join", (attn_join_kernel<D, NCP, NCO, kAtOnce>), dim3((unsigned)rows), dim3(256), 0, stream, a);
  else
    MOE_LAUNCH("attn_join", (attn_join_kernel<D, NCP, NCO, 1>), dim3((unsigned)((rows + kAtOnce - 1) / kAtOnce)), dim3(256), 0,
               stream, a);
  return check_launch("moe_attn_decode");
}

template <int D>
moe_status_t dispatch_decode(const DecodeArgs& a, const DecodePlan& p, hipStream_t stream) {
  if (p.own == 2) return launch_decode<D, 2, 2>(a, p, stream);
  return p.front == 1 ? launch_decode<D, 1, 1>(a, p, stream) : launch_decode<D, 2, 1>(a, p, stream);
}

}  // namespace

}  // namespace moe

using namespace moe;

extern "C" size_t moe_attn_decode_workspace(moe_attn_dims_t d, int32_t B, int32_t max_len, int32_t prefix_len) {
  if (check_attn_dims(d, "moe_attn_decode_workspace") != MOE_OK || B < 1 || B > 65535 || max_len < 0 || prefix_len < 0 ||
      max_len > kMostKeys || prefix_len > kMostKeys)
    return 0;
  return decode_workspace(d, B, max_len, prefix_len);
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
  if ((!page_table && table_width > 0) || !lens || !out || (prefix_len > 0 && !prefix_pages))
    return fail(MOE_ERR_INVALID_ARG, "moe_attn_decode: null pointer");
  if (!aligned(out, 16)) return fail(MOE_ERR_INVALID_ARG, "moe_attn_decode: out must be 16-byte aligned");
  const DecodePlan p = plan_decode(d, B, max_len, prefix_len);
  const int64_t row_keys = std::min<int64_t>((int64_t)table_width * cache.page_size, kMostKeys);
  if ((int64_t)p.prefix_blocks * steps_of(prefix_len) + (int64_t)p.own_blocks * B * steps_of((int)row_keys) > 0x7fffffff)
    return fail(MOE_ERR_UNSUPPORTED_SHAPE, "moe_attn_decode: %d sequences of %lld keys and a prefix of %d: over 2^31 steps", B,
                (long long)row_keys, prefix_len);
  const size_t need = p.bytes();
  if (need && (!ws || ws_bytes < need || !aligned(ws, 256)))
    return fail(MOE_ERR_WORKSPACE, "moe_attn_decode: workspace %zu bytes, needs %zu, 256-byte aligned", ws_bytes, need);
  uint8_t* base = static_cast<uint8_t*>(ws);
  DecodeArgs a{q, q_stride, cache, page_table, lens, prefix_pages, out, nullptr, nullptr, nullptr, dev_status, B,
               table_width, prefix_len, d.kv_heads, d.q_heads / d.kv_heads, __builtin_ctz((unsigned)cache.page_size),
               p.prefix_blocks, p.own_blocks, p.pieces, scale * kLog2e};
  if (need) {
    a.seg_o = reinterpret_cast<float*>(base);
    a.seg_ml = reinterpret_cast<float2*>(base + p.o_bytes);
    a.starts = reinterpret_cast<uint32_t*>(base + p.o_bytes + p.ml_bytes);
  }
  return d.head_dim == 64 ? dispatch_decode<64>(a, p, stream) : dispatch_decode<128>(a, p, stream);
}
