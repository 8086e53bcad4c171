// Attention over packed prompts.
//
// The rows of one product are the queries of a key/value head's whole group:
// row r of sequence b is token r / G, head r % G of the group (G = q_heads /
// kv_heads), so keys and values are read once for the group and a short chunk of
// tokens still fills a tile.  A workgroup takes a tile of rows and walks the
// keys in tiles of 64, staged through LDS; each wave has 32 rows and computes
// the transposed products with 32x32x16 bf16 MFMAs:
//   S^T = K Q^T   a lane holds one row's (lane % 32) scores of 16 of 32 keys, so
//                 the softmax's maximum and sum are in-lane but for one exchange
//                 between the half-waves, and m and l are one register each
//   O^T = V^T P^T the scores' registers are the second operand as they stand: a
//                 product's sum over keys may run in any order, and V's operand
//                 is read from LDS in the order that the scores have (8 s + 4 h +
//                 i for half-wave h), transposed by ds_read_b64_tr_b16.
// Sums are fp32; the numerators are rounded to bf16 for the second product, and
// the denominators are sums of the rounded ones, so that the weights still add up
// to 1 (error 2.0e-3 of the result's norm, 1.6e-3 of it the output's rounding).
//
// Bound by the matrix cores, 4 * head_dim flops per row and key, and by the power
// that they draw when all are busy (the clock falls to 1.6 - 2.0 GHz).  16384
// causal tokens of 32 heads of 128: 1.86 to 1.95 ms from card to card, 1130 to 1180
// TFLOP/s, where the largest library products reach 1340.  Eight prompts of 357 to
// 2048 tokens: 147 to 152 us, 810 to 830 TFLOP/s, the matrix cores busy for 41 % of
// the cycles; their 1248 workgroups of unequal length end unevenly, each with a
// beginning and an end that nothing covers.  Where there are fewer workgroups than
// CUs, a call takes 5 us and 1.4 us for each key tile of the longest rows: rows are
// then shared by two halves of a workgroup's waves, and keys cut into parts.  Heads
// of 64 are bound by the vector phase and by their longest rows (403 and 2995 tokens
// of 24 heads over 8: 60 us for 28 GFLOP).
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "attention.h"

namespace moe {

namespace {

struct PrefillArgs {
  const uint16_t *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;
  const int32_t *cu_q, *cu_k;
  uint16_t* out;
  float* part_o;   // [T_q * q_heads][parts][D]: a part's sums, not divided
  float* part_ml;  // [T_q * q_heads][parts][2]: its running maximum and sum (0: nothing in part_o)
  int32_t* status;
  int B, T_q, T_k, kv_heads, group, causal;
  uint32_t group_inverse;  // ceil(2^21 / group): n / group = n * group_inverse >> 21 for n < 1280, group <= 1024
  int parts, part_tiles;   // key tiles are cut into parts of this many, the last takes what is left
  float c;  // scale * log2(e): the softmax runs on powers of 2
  uint32_t looks;  // the workgroup that looks at the offsets
};

constexpr int kKeys = 64;  // keys per tile
constexpr int kRing = 4;   // tiles of keys, and of values, in LDS
constexpr int kWaveRows = 32;

// One row tile: its place in its sequence, the sequence's rows and keys, all the
// same for the workgroup and in scalar registers.
struct RowTile {
  int local, n_tiles;      // place, and the sequence's number of tiles
  int q0, lq, k0, lk;
};

// Reports offsets that leave the tensors or decrease, of sequences without rows too.
__device__ __forceinline__ void report_offsets(const PrefillArgs& a) {
  bool bad = false;
  for (int b = threadIdx.x; b < a.B; b += blockDim.x) {
    const int q_lo = a.cu_q[b], q_hi = a.cu_q[b + 1], k_lo = a.cu_k[b], k_hi = a.cu_k[b + 1];
    bad |= q_lo < 0 || q_hi > a.T_q || q_lo > q_hi || k_lo < 0 || k_hi > a.T_k || k_lo > k_hi;
  }
  if (__any(bad) && (threadIdx.x & 63) == 0) atomicOr(a.status, MOE_DEV_BAD_LENGTH);
}

// Row tile `tile`, counted over the sequences in order; false behind the last.
// Every lane of a wave calls it.  32 bits hold the counts: the launch checks
// that rows (T_q * group) and tiles do.
__device__ __forceinline__ bool find_tile(const PrefillArgs& a, int tile_rows, int tile, RowTile& r) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int base = 0; base < a.B; base += 64) {
    const int b = min(base + lane, a.B - 1);
    const int q_lo = a.cu_q[b], q_hi = a.cu_q[b + 1], k_lo = a.cu_k[b], k_hi = a.cu_k[b + 1];
    const int q0 = min(max(q_lo, 0), a.T_q), k0 = min(max(k_lo, 0), a.T_k);
    const int lq = base + lane < a.B ? max(min(max(q_hi, 0), a.T_q) - q0, 0) : 0;
    const int lk = max(min(max(k_hi, 0), a.T_k) - k0, 0);
    const int n = (int)(((uint32_t)lq * a.group + tile_rows - 1) / tile_rows);
    const int incl = wave_scan(n);
    const uint64_t past = __ballot(before + incl > tile);
    if (past) {
      const int w = __ffsll((unsigned long long)past) - 1;
      r.n_tiles = __builtin_amdgcn_readlane(n, w);
      r.local = tile - before - (__builtin_amdgcn_readlane(incl, w) - r.n_tiles);
      r.q0 = __builtin_amdgcn_readlane(q0, w);
      r.lq = __builtin_amdgcn_readlane(lq, w);
      r.k0 = __builtin_amdgcn_readlane(k0, w);
      r.lk = __builtin_amdgcn_readlane(lk, w);
      return true;
    }
    before += __builtin_amdgcn_readlane(incl, 63);
  }
  return false;
}

// LDS place of 16-byte chunk c of a staged row (256 bytes at D = 128, 128 at
// D = 64).  The xor spreads the rows that one instruction reads over the 256
// bytes of the banks: 16 rows at one chunk (an operand of K), or 4 rows at 4
// neighbouring chunks (transposed reads of V).
template <int D>
__device__ __forceinline__ int staged(int row, int c) {
  const int f = D == 128 ? ((row & 3) << 2) | ((row >> 2) & 3) : ((row & 2) << 1) | ((row >> 2) & 3);
  return row * (D * 2) + ((c ^ f) * 16);
}

// 1 KB a wave straight into LDS, from base + offset (base uniform, offset the
// lane's).  A vector memory instruction needs five wait states after a vector
// instruction wrote its scalar base.
__device__ __forceinline__ void async_load_1k_at(const void* base, uint32_t offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(__builtin_amdgcn_readfirstlane((int)lds)), "v"(offset), "s"(base)
               : "memory");
}

// The maximum over a lane and lane ^ 32, by a register swap between the half-waves.
__device__ __forceinline__ float pair_max(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}

// One wave's part of staging keys or values t0 .. t0 + 63: 1 KB a call, straight
// into LDS, in the order that `staged` gives (a lane fetches the chunk that
// belongs at its place).  Rows behind the sequence's end repeat its last:
// finite, weighed by 0.
template <int D, int WAVES>
__device__ __forceinline__ void stage(const uint16_t* base, int64_t stride, int t0, int last, int wave, uint32_t lds) {
  constexpr int kCalls = kKeys * D * 2 / 1024 / WAVES, kRows = 1024 / (D * 2);
  const int lane = threadIdx.x & 63;
  t0 = min(t0, last);
  const uint16_t* tile = base + t0 * stride;
#pragma unroll
  for (int i = 0; i < kCalls; ++i) {
    const int call = wave * kCalls + i;
    const int row = call * kRows + lane / (D / 8);
    const int c = (staged<D>(row, lane % (D / 8)) % (D * 2)) / 16;
    // a row's offset in its tile has 30 bits: strides have 24 in bytes
    async_load_1k_at(tile, __umul24(min(row, last - t0), (uint32_t)(stride * 2)) + 16 * c, lds + 1024 * call);
  }
}

// kSplit: the two halves of the waves take the same rows, one the even key tiles
// and the other the odd ones, and their sums are joined at the end: half the rows
// a workgroup and half the steps, for launches that leave CUs without work.
template <int D, int WAVES, bool kSplit>
__global__ __launch_bounds__(64 * WAVES, 2) void attn_prefill_kernel(PrefillArgs a) {
  constexpr int kHalf = WAVES / 2;
  constexpr int kTileRows = kWaveRows * (kSplit ? kHalf : WAVES), kTileBytes = kKeys * D * 2;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[2][kRing][kTileBytes];  // keys, values
  __shared__ __attribute__((aligned(1024))) uint8_t late_q[kHalf * kWaveRows * D * 2];

  // With a status word the grid has one workgroup more, which looks at the offsets (a sequence that is cut to nothing has
  // no tile, and the tiles' workgroups need not look behind theirs).
  if (blockIdx.x == a.looks) {
    report_offsets(a);
    return;
  }
  const uint32_t item = blockIdx.x / (uint32_t)a.kv_heads;
  const int kvh = blockIdx.x - item * a.kv_heads, tile = item / (uint32_t)a.parts, part = item - tile * a.parts;
  RowTile rt;
  if (!find_tile(a, kTileRows, tile, rt)) return;
  const int q0 = rt.q0, lq = rt.lq, k0 = rt.k0, lk = rt.lk;

  const int lane = threadIdx.x & 63, col = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool late = wave >= kHalf;
  const int wave_row = kWaveRows * (kSplit && late ? wave - kHalf : wave);  // of the tile, the wave's first
  const uint32_t group = a.group, n_rows = (uint32_t)lq * group;
  const uint32_t row0 = (uint32_t)(rt.n_tiles - 1 - rt.local) * kTileRows;  // a sequence's longest rows first
  // row i of the tile, i < kTileRows: its token and head (rows behind the sequence's last are that row)
  const uint32_t tok0 = row0 / group, head0 = row0 - tok0 * group, last_row = min((uint32_t)kTileRows, n_rows - row0) - 1;
  const auto row_of = [&](uint32_t i, int& tok, int& head) __attribute__((always_inline)) {
    const uint32_t n = head0 + min(i, last_row), t = n * a.group_inverse >> 21;
    tok = tok0 + t;
    head = kvh * group + (n - t * group);
  };
  int tok, head;
  row_of(wave_row + col, tok, head);
  const bool live = (uint32_t)(wave_row + col) <= last_row;
  // the last key that this row sees, that the tile's first row sees and that its last row sees
  int limit = min(a.causal ? tok + lk - lq : lk - 1, lk - 1);
  const int first_limit = min(a.causal ? (int)tok0 + lk - lq : lk - 1, lk - 1);
  const int tile_last = a.causal ? (int)((row0 + last_row) / group) + lk - lq : lk - 1;
  const int n_key_tiles = tile_last < 0 ? 0 : tile_last / kKeys + 1;
  // this part's tiles
  const int kt0 = min(part * a.part_tiles, n_key_tiles);
  const int kt1 = part == a.parts - 1 ? n_key_tiles : min(kt0 + a.part_tiles, n_key_tiles);
  if (kSplit) limit = min(limit, kt1 * kKeys - 1);  // one half may take a tile behind the last

  v16f o[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) o[i] = v16f{};
  float m = kNoScore;
  // Denominators, the sums of the rounded numerators.  D = 64, whose vector phase is the longer one: by a product with ones
  // more for every 16 keys, in all 16 of `total` (two prompts of up to 2995 tokens, 24 heads: 59.5 us, 61.5 by dot
  // products).  D = 128: by a dot product with ones for every two of the lane's keys, in total[0] and total[1] (16384
  // tokens, 32 heads: 1991 us, 2046 by the product).
  constexpr bool kSumByProduct = D == 64;
  v16f total{};

  if (kt0 < kt1) {
    const uint16_t* kbase = a.k + (int64_t)k0 * a.k_stride + kvh * D;
    const uint16_t* vbase = a.v + (int64_t)k0 * a.v_stride + kvh * D;
    const uint32_t lds0 = lds_address(lds);
    const auto fetch_k = [&](int kt) __attribute__((always_inline)) {
      stage<D, WAVES>(kbase, a.k_stride, kt * kKeys, lk - 1, wave, lds0 + kt % kRing * kTileBytes);
    };
    const auto fetch_v = [&](int kt) __attribute__((always_inline)) {
      stage<D, WAVES>(vbase, a.v_stride, kt * kKeys, lk - 1, wave, lds0 + (kRing + kt % kRing) * kTileBytes);
    };
    constexpr int kCalls = 2 * (kTileBytes / 1024 / WAVES);  // of a wave for one tile's keys and values

    v8bf qf[D / 16];  // the row's query
    v16f s[2];        // scores of a tile
    union {
      v8bf v[4];
      uint32_t x[16];
    } p;              // its numerators

    // Operand f of a step: the next tile's keys (the first D / 8, the two blocks of 32 keys in turn), then this tile's
    // values.  The swizzle makes an operand's place the first one's with some bits flipped, plus a constant.
    constexpr int kK = D / 8, kAhead = 6;
    const int k_place = lds0 + staged<D>(col, h);
    // lane j of a 16-lane group gives the address of row j / 4, 8-byte piece j % 4 of a 4 x 16 block and gets column j
    const int v_place = lds0 + kRing * kTileBytes +
                        staged<D>(4 * h + ((lane & 15) >> 2), 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) + 8 * (lane & 1);
    const auto operand = [&](int kp, int vp, int f) __attribute__((always_inline)) {
      union {
        v8bf v;
        v4s x[2];
      } r;
      if (f < kK) {
        r.v = *(__attribute__((address_space(3))) const v8bf*)(uintptr_t)((kp ^ (32 * (f >> 1))) + (f & 1) * 32 * (D * 2));
        return r.v;
      }
      const int w = (f - kK) / (D / 32), dt = (f - kK) % (D / 32);
#pragma unroll
      for (int x = 0; x < 2; ++x)
        r.x[x] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(uintptr_t)(
            (vp ^ (64 * dt + 32 * x)) + (16 * w + 8 * x) * (D * 2)));
      return r.v;
    };
    // The vector phase of tile kt: its scores become numerators; maximum, sum and accumulator follow.  A tile behind
    // the row's last key changes nothing (masked).
    const auto weigh = [&](auto masked, int kt) __attribute__((always_inline)) {
      if (decltype(masked)::value) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (kt * kKeys + 32 * u + 8 * (i / 4) + 4 * h + (i & 3) > limit) s[u][i] = -INFINITY;
      }
      float top = s[0][0];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, s[u][i]);
      top = pair_max(top) * a.c;
      // The accumulator is rescaled only when some row's maximum has grown by more than 2^8: numerators up to 2^8 are
      // as exact, and most tiles of a long row go without.
      if (__any(top > m + 8.0f)) {
        const float m_new = fmaxf(m, top), alpha = __builtin_amdgcn_exp2f(m - m_new);
        m = m_new;
        if (kSumByProduct) {
          total *= alpha;
        } else {
          total[0] *= alpha;
          total[1] *= alpha;
        }
#pragma unroll
        for (int i = 0; i < D / 32; ++i) o[i] *= alpha;
      }
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
          const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][i], a.c, -m));
          const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][i + 1], a.c, -m));
          p.x[8 * u + i / 2] = pack_bf16(x, y);
          if (!kSumByProduct) {
            const v2bf pair = {p.v[2 * u + i / 8][i % 8], p.v[2 * u + i / 8][i % 8 + 1]}, one = {(__bf16)1.0f, (__bf16)1.0f};
            total[u] = __builtin_amdgcn_fdot2_f32_bf16(pair, one, total[u], false);
          }
        }
    };
    // A step is a vector phase (`weigh`) and a matrix phase: the next tile's scores, then this tile's numerators times
    // its values, with the operands read from LDS kAhead products early, the first ones before the phase begins.
    //
    // The two waves of a SIMD run a phase apart, so that one has matrix work while the other has vector work: the
    // late half of the waves starts with one barrier more.  In phase 2 t the early half multiplies tile t and the late
    // half weighs it; in phase 2 t + 1 the early half weighs tile t + 1 and the late half multiplies tile t.
    //
    // Ring: keys t and values t - 1 are last read in phase 2 t - 1 (by the late half's matrix phase of tile t - 1).  Keys
    // t + kRing and values t + kRing - 1 take their places, fetched in phase 2 t by the late half and in phase 2 t + 1 by
    // the early one, at the start of their vector phases.  They are first read at the end of phase 2 (t + kRing) - 3.
    // Every vector phase ends by waiting for all fetches but its own, so a fetch has two phases or more to
    // arrive, and the barrier after that wait comes before the first read.  (The scores of the tile behind the last are
    // not used.)
    //
    // kSplit: phase t multiplies tile t, in the early half for even t (counted from kt0) and in the late one for odd t,
    // while the other half weighs tile t + 1.  Keys t + 2 and values t are read in phase t (the first of those keys at the
    // end of phase t - 1) and by nothing else.  Both halves fetch keys t + 5 and values t + 3 at the start of phase t, to
    // the places of keys t + 1 and values t - 1, and every phase ends by waiting for all fetches but its own: they have two
    // phases to arrive, and keys t + 5 one more before the end of phase t + 2.
    const int end = kSplit ? kt0 + ((kt1 - kt0 + 1) & ~1) : kt1;  // kSplit: both halves take as many steps
    v8bf ones;
#pragma unroll
    for (int i = 0; i < 8; ++i) ones[i] = (__bf16)1.0f;
    const auto step = [&](auto masked, int kt) __attribute__((always_inline)) {
      constexpr int kNext = kSplit ? 2 : 1;  // the half's next tile
      const int ft = kSplit || late ? kt : kt - 1;
      // nothing behind the end, but where the branch costs more (kSplit: two prompts of up to 1950 tokens 32.7 us without,
      // 34.8 with)
      const bool more = kSplit || ft + kRing - kNext < end;
      if (more) {
        fetch_k(ft + kRing);
        fetch_v(ft + kRing - kNext);
      }
      weigh(masked, kt);
      // opaque: the operands' places are computed in every step, which costs less than the registers to keep them
      int kp = k_place + (kt + kNext) % kRing * kTileBytes, vp = v_place + kt % kRing * kTileBytes;
      asm volatile("" : "+v"(kp), "+v"(vp));
      v8bf ops[kAhead + 1];
#pragma unroll
      for (int f = 0; f < kAhead; ++f) ops[f] = operand(kp, vp, f);
      __builtin_amdgcn_sched_barrier(0);
      if (!more) asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
      asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" : : "n"(kCalls) : "memory");
      if (kSplit) {
        fetch_k(kt + kRing + 1);
        fetch_v(kt + kRing - 1);
      }
      __builtin_amdgcn_s_setprio(1);
      __builtin_amdgcn_sched_barrier(0);
      s[0] = s[1] = v16f{};
#pragma unroll
      for (int f = 0; f < 2 * kK; ++f) {
        if (f + kAhead < 2 * kK) ops[(f + kAhead) % (kAhead + 1)] = operand(kp, vp, f + kAhead);
        const v8bf x = ops[f % (kAhead + 1)];
        const int g = f - kK;
        if (f < kK)
          s[f & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, qf[f >> 1], s[f & 1], 0, 0, 0);
        else
          o[g % (D / 32)] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, p.v[g / (D / 32)], o[g % (D / 32)], 0, 0, 0);
        if (kSumByProduct && f >= kK && g % (D / 32) == 0)
          total = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ones, p.v[g / (D / 32)], total, 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
      __builtin_amdgcn_s_setprio(0);
      if (kSplit)
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" : : "n"(kCalls) : "memory");
      else
        asm volatile("s_barrier" : : : "memory");
      __builtin_amdgcn_sched_barrier(0);
    };

    // The wave's rows of queries come the way that keys do, whole rows straight into LDS (the early half's into the places
    // of values kt0 + 2 and kt0 + 3, the late one's into a place of their own), and from there as operands.
    constexpr int kQBytes = kWaveRows * D * 2;
    static_assert(kHalf * kQBytes == 2 * kTileBytes, "half the waves' queries are two tiles");
    const int q_lds = late ? lds_address(late_q) + (wave - kHalf) * kQBytes
                           : lds0 + (kRing + (kt0 + 2 + wave / 2) % kRing) * kTileBytes + (wave & 1) * kQBytes;
    constexpr int kQCalls = kWaveRows * D * 2 / 1024;
#pragma unroll
    for (int i = 0; i < kQCalls; ++i) {
      const int row = i * (kWaveRows / kQCalls) + lane / (D / 8);
      const int c = (staged<D>(row, lane % (D / 8)) % (D * 2)) / 16;
      int t, hd;
      row_of(wave_row + row, t, hd);
      async_load_1k(a.q + (int64_t)(q0 + t) * a.q_stride + hd * D + 8 * c, q_lds + 1024 * i);
    }
    fetch_k(kt0);
    fetch_k(kt0 + 1);
    fetch_k(kt0 + 2);
    fetch_v(kt0);
    fetch_v(kt0 + 1);
    if (kSplit) fetch_k(kt0 + 3);
    // queries, keys kt0 and keys kt0 + 1
    asm volatile("s_waitcnt vmcnt(%0)" : : "n"(kSplit ? 2 * kCalls : 3 * kCalls / 2) : "memory");
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
      qf[i] = *(__attribute__((address_space(3))) const v8bf*)(uintptr_t)(q_lds + staged<D>(col, 2 * i + h));
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
    const int first = kSplit && late ? kt0 + 1 : kt0;  // the half's first tile
    s[0] = s[1] = v16f{};
#pragma unroll
    for (int f = 0; f < kK; ++f)
      s[f & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(operand(k_place + first % kRing * kTileBytes, v_place, f), qf[f >> 1],
                                                         s[f & 1], 0, 0, 0);
    // keys kt0 and kt0 + 1 have been read, and keys kt0 + 2 are there
    if (kSplit) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(3 * kCalls / 2) : "memory");
    if (late) {
      fetch_k(kSplit ? kt0 + kRing : kt0 + kRing - 1);
      fetch_v(kt0 + kRing - 2);
      asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" : : "n"(kCalls) : "memory");
    }
    const int n_free = min((first_limit + 1) / kKeys, kt1);  // tiles before it have no masked key for any row
    int kt = first;
    for (; kt < min(n_free, end); kt += kSplit ? 2 : 1) step(std::false_type{}, kt);
    for (; kt < end; kt += kSplit ? 2 : 1) step(std::true_type{}, kt);
    if (!late) asm volatile("s_barrier" : : : "memory");
    wait_async_and_barrier<0>();  // no fetch is on its way to LDS, and no wave reads from it any more

    // A product multiplies a hidden key's value by 0, which an infinite or NaN value does not survive.  If a sum is not
    // finite, the wave takes its sums again; maxima and denominators stand.  Tiles that all its rows see whole are products
    // as before, their operands straight from memory; in the others every key is weighed for the rows that see it alone.
    // 16384 tokens of 32 heads of 128 with an infinite value that all rows see: 9.6 ms (164 key by key), 2.2 without.
    float finite = 0.0f;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) finite = fmaf(o[i][j], 0.0f, finite);
    if (__any(finite != 0.0f)) {
#pragma unroll
      for (int i = 0; i < D / 32; ++i) o[i] = v16f{};
      int tile = first;
#pragma unroll 1
      for (; tile < n_free; tile += kSplit ? 2 : 1) {
        s[0] = s[1] = v16f{};
#pragma unroll
        for (int f = 0; f < kK; ++f) {
          const int64_t key = tile * kKeys + 32 * (f & 1) + col;
          const v8bf x = *reinterpret_cast<const v8bf*>(kbase + key * a.k_stride + 16 * (f >> 1) + 8 * h);
          s[f & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, qf[f >> 1], s[f & 1], 0, 0, 0);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int i = 0; i < 16; i += 2)
            p.x[8 * u + i / 2] = pack_bf16(__builtin_amdgcn_exp2f(__builtin_fmaf(s[u][i], a.c, -m)),
                                           __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][i + 1], a.c, -m)));
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
          for (int dt = 0; dt < D / 32; ++dt) {
            union {
              v8bf v;
              uint16_t x[8];
            } y;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const int64_t key = tile * kKeys + 16 * w + 8 * (e / 4) + 4 * h + (e & 3);
              y.x[e] = vbase[key * a.v_stride + 32 * dt + col];
            }
            o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(y.v, p.v[w], o[dt], 0, 0, 0);
          }
      }
#pragma unroll 1
      for (; tile < kt1; tile += kSplit ? 2 : 1)
#pragma unroll 1
        for (int j0 = tile * kKeys; j0 <= min(tile * kKeys + kKeys - 1, tile_last); j0 += 4)  // four on their way at once
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const int64_t j = min(j0 + x, tile_last);  // (limit <= tile_last)
            const bool sees = j0 + x <= limit;
            float score = 0.0f;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
              const v8bf key = *reinterpret_cast<const v8bf*>(kbase + j * a.k_stride + 16 * i + 8 * h);
#pragma unroll
              for (int e = 0; e < 8; ++e) score = fmaf((float)qf[i][e], (float)key[e], score);
            }
            score += __shfl_xor(score, 32, 64);
            const float w = (float)(__bf16)__builtin_amdgcn_exp2f(fmaf(score, a.c, -m));
#pragma unroll
            for (int i = 0; i < D / 8; ++i) {
              const uint2 y = *reinterpret_cast<const uint2*>(vbase + j * a.v_stride + 8 * i + 4 * h);
              const float v[4] = {__uint_as_float(y.x << 16), __uint_as_float(y.x & 0xffff0000u), __uint_as_float(y.y << 16),
                                  __uint_as_float(y.y & 0xffff0000u)};
#pragma unroll
              for (int e = 0; e < 4; ++e) o[i / 4][4 * (i % 4) + e] += sees ? w * v[e] : 0.0f;
            }
          }
    }
  }

  float l = total[0];
  if (!kSumByProduct) {
    l += total[1];
    l += __shfl_xor(l, 32, 64);
  }
  if (kSplit) {
    // the late half's sums by way of LDS to the early half, lane by lane
    float2* late_ml = reinterpret_cast<float2*>(late_q) + (wave & (kHalf - 1)) * 64 + lane;
    v4f* late_o = reinterpret_cast<v4f*>(&lds[0][0][0] + (wave & (kHalf - 1)) * (kWaveRows * D * 4)) + lane;
    if (late) {
      *late_ml = make_float2(m, l);
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) late_o[64 * (4 * i + j)] = v4f{o[i][4 * j], o[i][4 * j + 1], o[i][4 * j + 2], o[i][4 * j + 3]};
    }
    __syncthreads();
    if (late) return;
    const float2 ml = *late_ml;
    const float top = fmaxf(m, ml.x), f = __builtin_amdgcn_exp2f(m - top), e = __builtin_amdgcn_exp2f(ml.x - top);
    m = top;
    l = l * f + ml.y * e;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const v4f x = late_o[64 * (4 * i + j)];
#pragma unroll
        for (int k = 0; k < 4; ++k) o[i][4 * j + k] = o[i][4 * j + k] * f + x[k] * e;
      }
  }
  // Whole rows go out: a lane has pieces of 4 elements of one row, which the wave's part of LDS turns into rows (with
  // stores of 16 or 32 bytes a row the eight prompts took 168 us, with whole rows in and out 152).
  const int64_t heads = a.kv_heads * group;
  uint8_t* turn = &lds[0][0][0] + wave * (2 * kRing * kTileBytes / WAVES);
  if (a.parts > 1) {
    const int64_t row = (q0 + (int64_t)tok) * heads + head;
    if (live && h == 0) *reinterpret_cast<float2*>(a.part_ml + (row * a.parts + part) * 2) = make_float2(m, l);
    if (kt0 >= kt1) return;
    constexpr int kPieces = D / 4;  // of 16 bytes
    static_assert(kWaveRows * D * 4 <= 2 * kRing * kTileBytes / WAVES, "a wave's rows in fp32 fit its part of LDS");
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4*>(turn + col * (D * 4) + (((8 * dt + 2 * i + h) ^ (col & 15)) * 16)) =
            make_float4(o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]);
#pragma unroll
    for (int i = 0; i < kWaveRows * kPieces / 64; ++i) {
      const int at = 64 * i + lane, rr = at / kPieces, c = at % kPieces;
      if ((uint32_t)(wave_row + rr) > last_row) continue;
      int t, hd;
      row_of(wave_row + rr, t, hd);
      *reinterpret_cast<float4*>(a.part_o + (((q0 + (int64_t)t) * heads + hd) * a.parts + part) * D + 4 * c) =
          *reinterpret_cast<const float4*>(turn + rr * (D * 4) + ((c ^ (rr & 15)) * 16));
    }
    return;
  }
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
  constexpr int kPieces = D / 8;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<uint2*>(turn + staged<D>(col, 4 * dt + i) + 8 * h) =
          make_uint2(pack_bf16(o[dt][4 * i] * inv, o[dt][4 * i + 1] * inv),
                     pack_bf16(o[dt][4 * i + 2] * inv, o[dt][4 * i + 3] * inv));
#pragma unroll
  for (int i = 0; i < kWaveRows * kPieces / 64; ++i) {
    const int at = 64 * i + lane, rr = at / kPieces, c = at % kPieces;
    if ((uint32_t)(wave_row + rr) > last_row) continue;
    int t, hd;
    row_of(wave_row + rr, t, hd);
    *reinterpret_cast<uint4*>(a.out + ((q0 + (int64_t)t) * heads + hd) * D + 8 * c) =
        *reinterpret_cast<const uint4*>(turn + staged<D>(rr, c));
  }
}

// The parts' sums of a row, weighed by their maxima: D / 4 lanes a row, 16 bytes
// each.  Rows outside all sequences have no parts and are left alone.
template <int D>
__global__ __launch_bounds__(256) void attn_prefill_join_kernel(PrefillArgs a, int64_t n_rows) {
  const int64_t row = (int64_t)blockIdx.x * (256 / (D / 4)) + threadIdx.x / (D / 4);
  const int d = threadIdx.x % (D / 4) * 4;
  if (row >= n_rows) return;
  const int64_t t = row / (a.kv_heads * a.group);
  if (t < a.cu_q[0] || t >= a.cu_q[a.B]) return;
  const float2* ml = reinterpret_cast<const float2*>(a.part_ml) + row * a.parts;
  float m = kNoScore, l = 0.0f;
  v4f o = {};
  // Eight parts at a time, all on their way before the first is used (16 parts of few rows: 10.9 us with one behind the
  // other, 4.0 with eight).
  constexpr int kBatch = 8;
  for (int p = 0; p < a.parts; p += kBatch) {
    float2 x[kBatch];
    v4f part[kBatch];
    float top = m;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      x[i] = make_float2(kNoScore, 0.0f);
      part[i] = v4f{};
      if (p + i < a.parts) {
        x[i] = ml[p + i];
        part[i] = *reinterpret_cast<const v4f*>(a.part_o + (row * a.parts + p + i) * D + d);
      }
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) top = fmaxf(top, x[i].x);
    const float f = __builtin_amdgcn_exp2f(m - top);
    m = top;
    l *= f;
    o *= f;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const bool there = x[i].y != 0.0f;  // a part without keys has written no sums; one with NaN keeps it
      const float e = there ? __builtin_amdgcn_exp2f(x[i].x - m) : 0.0f;
      l += x[i].y * e;
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] += there ? part[i][j] * e : 0.0f;
    }
  }
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
  *reinterpret_cast<uint2*>(a.out + row * D + d) =
      make_uint2(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv));
}

constexpr int kWaves = 8;

struct PrefillPlan {
  int64_t tiles;  // bound on the row tiles
  bool split;     // waves of a workgroup share rows
  int parts, part_tiles;
  size_t o_bytes, ml_bytes;
};

// The height of the row tiles and the number of parts that the keys are cut into:
// those whose estimated time is the least.  A CU runs one workgroup at a time; one
// takes about 5 us and a step for each of its key tiles, or 6.3 us and a longer
// step for each two of them (a step takes a third longer than assumed where all CUs
// are busy: the 34 tiles of a part below 72 us, not 54).  Joining parts costs a launch, 4.5 us, and their sums go
// to memory and back at about 4 TB/s.  Whole rows against halves: 1040 tokens of 16
// heads of 64 23.7 and 17.1 us, 206 tokens of 40 heads over 8 of 128 behind 320
// keys 18.5 and 15.5; where the card is full, eight prompts of up to 2048 tokens,
// 157 and 208 (twice the keys go through LDS).  509 tokens of 32 heads over 8
// behind 8192 keys are 64 workgroups of 136 tiles: 184 us whole, 72 us in four
// parts and 8 us to join them.
//
// What the chosen number of parts needs goes up and down with the sizes, and a
// caller has one workspace for calls of many sizes.  So the plan keeps to
// `most_sums`, which only grows, and a call that cuts its keys asks for all of that.
constexpr double kStart[2] = {5.0, 6.3};  // us of a workgroup, whole rows and shared ones
double step_us(int32_t head_dim, int split) { return head_dim == 128 ? (split ? 1.8 : 1.45) : (split ? 1.25 : 1.1); }
constexpr int kMostParts = 16;

// Bytes of the parts' sums that a call of these sizes or smaller ones may use.  More parts than key tiles are never
// faster; and the sums' way to memory and back, 8 bytes an element at 4 TB/s, takes less than what parts can save, which
// is one round of workgroups (kStart + step_us for each key tile): bytes < 2e6 of the us of a round.  Half of that has
// been enough for every plan of 14 head layouts, 1 to 300 sequences, up to 60000 tokens and 10^6 keys (0.43 at the most).
size_t most_sums(const moe_attn_dims_t& d, int32_t T_q, int32_t max_k) {
  const int key_tiles = max_k / kKeys + 1;
  if (key_tiles == 1) return 0;
  const size_t each = (size_t)T_q * d.q_heads * d.head_dim * sizeof(float) * std::min(kMostParts, key_tiles);
  return std::min(each, (size_t)(1e6 * (kStart[0] + step_us(d.head_dim, 0) * key_tiles)));
}

PrefillPlan plan_prefill(const moe_attn_dims_t& d, int32_t B, int32_t T_q, int32_t max_k) {
  PrefillPlan p{};
  const int group = d.q_heads / d.kv_heads;
  const int64_t rows = (int64_t)T_q * d.q_heads;
  const int key_tiles = max_k / kKeys + 1;
  const size_t most = most_sums(d, T_q, max_k);
  // a causal prompt's rows see the keys before them: their mean over the longest's
  const double mean = 1.0 - std::min((double)T_q / B, (double)max_k) / (2.0 * std::max(max_k, 1)), even = 2.0 * mean - 1.0;
  double best = 0.0;
  for (int split = 0; split < 2; ++split) {
    const int64_t tiles = (int64_t)T_q * group / (kWaves * kWaveRows >> split) + B;  // sequences may each add a part of one
    for (int parts = 1; parts <= std::min(kMostParts, key_tiles); ++parts) {
      if (parts > 1 && (size_t)rows * parts * d.head_dim * sizeof(float) > most) break;
      const int part_tiles = (key_tiles + parts - 1) / parts;
      const double steps = (part_tiles + split) >> split;
      // workgroups a CU: the more alike they are, the more a last round of few costs a whole one
      const double load = (double)(tiles * d.kv_heads * parts) / 256;
      const double rounds = load + (std::max(1.0, ceil(load)) - load) * even * even;
      const double start = kStart[split], step = step_us(d.head_dim, split);
      double us = std::max(start + step * steps, rounds * (start + step * steps * mean));
      if (parts > 1) us += 4.5 + (double)rows * parts * d.head_dim * 8 / 4e6;
      if (p.parts == 0 || us < best) {
        best = us;
        p.tiles = tiles;
        p.split = split != 0;
        p.parts = parts;
        p.part_tiles = part_tiles;
      }
    }
  }
  if (p.parts > 1) {
    p.o_bytes = ((size_t)rows * p.parts * d.head_dim * sizeof(float) + 255) & ~(size_t)255;
    p.ml_bytes = ((size_t)rows * p.parts * 2 * sizeof(float) + 255) & ~(size_t)255;
  }
  return p;
}

// A call's workspace where its plan has parts: sums, and a maximum and a sum for every head_dim of them.
size_t prefill_workspace(const moe_attn_dims_t& d, int32_t T_q, int32_t max_k) {
  const size_t sums = most_sums(d, T_q, max_k), pairs = sums / d.head_dim * 2;
  return ((sums + 255) & ~(size_t)255) + ((pairs + 255) & ~(size_t)255);
}

template <int D>
moe_status_t launch_prefill(PrefillArgs a, const PrefillPlan& p, hipStream_t stream) {
  // Heads fastest: workgroups that share keys have numbers equal mod 8 (one XCD's L2) where kv_heads is a multiple of
  // 8, and all heads' longest rows come first.
  const int64_t items = p.tiles * a.parts * a.kv_heads, rows = (int64_t)a.T_q * a.kv_heads * a.group;
  constexpr int kJoinRows = 256 / (D / 4);
  if ((items + 1) * kWaves * 64 >= (int64_t)1 << 32 || (rows / kJoinRows + 1) * 256 >= (int64_t)1 << 32)
    return fail(MOE_ERR_UNSUPPORTED_SHAPE, "moe_attn_prefill: %lld row tiles", (long long)items);
  const dim3 grid((unsigned)items + (a.status ? 1 : 0));
  a.looks = a.status ? (uint32_t)items : ~0u;
  if (p.split)
    MOE_LAUNCH("attn_prefill", (attn_prefill_kernel<D, kWaves, true>), grid, dim3(64 * kWaves), 0, stream, a);
  else
    MOE_LAUNCH("attn_prefill", (attn_prefill_kernel<D, kWaves, false>), grid, dim3(64 * kWaves), 0, stream, a);
  if (a.parts > 1)
    MOE_LAUNCH("attn_prefill_join", attn_prefill_join_kernel<D>, dim3((unsigned)((rows + kJoinRows - 1) / kJoinRows)),
               dim3(256), 0, stream, a, rows);
  return check_launch("moe_attn_prefill");
}

}  // namespace

}  // namespace moe

using namespace moe;

extern "C" size_t moe_attn_prefill_workspace(moe_attn_dims_t d, int32_t B, int32_t T_q, int32_t max_k) {
  if (check_attn_dims(d, "moe_attn_prefill_workspace") != MOE_OK || B < 1 || T_q < 1 || max_k < 0) return 0;
  return prefill_workspace(d, T_q, max_k);
}

extern "C" moe_status_t moe_attn_prefill(moe_attn_dims_t d, int32_t B, int32_t T_q, int32_t T_k, int32_t max_k,
                                         const uint16_t* q, int64_t q_stride, const uint16_t* k, int64_t k_stride,
                                         const uint16_t* v, int64_t v_stride, const int32_t* cu_q, const int32_t* cu_k,
                                         float scale, int32_t causal, uint16_t* out, int32_t* dev_status, void* ws,
                                         size_t ws_bytes, hipStream_t stream) {
  moe_status_t st = check_attn_dims(d, "moe_attn_prefill");
  if (st != MOE_OK) return st;
  if (B < 0 || T_q < 0 || T_k < 0 || max_k < 0)
    return fail(MOE_ERR_INVALID_ARG, "moe_attn_prefill: B=%d T_q=%d T_k=%d max_k=%d", B, T_q, T_k, max_k);
  if (!(scale > 0.0f) || !isfinite(scale * kLog2e)) return fail(MOE_ERR_INVALID_ARG, "moe_attn_prefill: scale=%g", scale);
  if (T_k > 1 << 30) return fail(MOE_ERR_UNSUPPORTED_SHAPE, "moe_attn_prefill: T_k=%d is over 2^30", T_k);
  if (B == 0 || T_q == 0) return MOE_OK;
  if ((st = check_rows(q, q_stride, d.q_heads, d.head_dim, "moe_attn_prefill", "q")) != MOE_OK) return st;
  if (T_k > 0 && (st = check_rows(k, k_stride, d.kv_heads, d.head_dim, "moe_attn_prefill", "k")) != MOE_OK) return st;
  if (T_k > 0 && (st = check_rows(v, v_stride, d.kv_heads, d.head_dim, "moe_attn_prefill", "v")) != MOE_OK) return st;
  if (!cu_q || !cu_k || !out) return fail(MOE_ERR_INVALID_ARG, "moe_attn_prefill: null pointer");
  if (!aligned(out, 16)) return fail(MOE_ERR_INVALID_ARG, "moe_attn_prefill: out must be 16-byte aligned");
  const PrefillPlan p = plan_prefill(d, B, T_q, max_k);
  const size_t need = p.parts > 1 ? prefill_workspace(d, T_q, max_k) : 0;
  if (need && (!ws || ws_bytes < need || !aligned(ws, 256)))
    return fail(MOE_ERR_WORKSPACE, "moe_attn_prefill: workspace %zu bytes, needs %zu, 256-byte aligned", ws_bytes, need);
  uint8_t* base = static_cast<uint8_t*>(ws);
  const PrefillArgs a{q, k, v, q_stride, k_stride, v_stride, cu_q, cu_k, out,
                      p.parts > 1 ? reinterpret_cast<float*>(base) : nullptr,
                      p.parts > 1 ? reinterpret_cast<float*>(base + p.o_bytes) : nullptr, dev_status,
                      B, T_q, T_k, d.kv_heads, d.q_heads / d.kv_heads, causal != 0,
                      (uint32_t)(((1 << 21) + d.q_heads / d.kv_heads - 1) / (d.q_heads / d.kv_heads)), p.parts, p.part_tiles,
                      scale * kLog2e, ~0u};
  return d.head_dim == 64 ? launch_prefill<64>(a, p, stream) : launch_prefill<128>(a, p, stream);
}
