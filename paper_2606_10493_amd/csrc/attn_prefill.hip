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
#include <math.h>

#include <algorithm>

#include "attention.h"

namespace moe {

namespace {

struct PrefillArgs {
  const uint16_t *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;
  const int32_t *cu_q, *cu_k;
  uint16_t* out;
  int32_t* status;
  int B, T_q, T_k, kv_heads, group, causal;
  float c;  // scale * log2(e): the softmax runs on powers of 2
};

constexpr int kKeys = 64;  // keys per tile
constexpr int kWaveRows = 32;

// Sequence b's rows of a packed tensor, cut to the tensor.
__device__ __forceinline__ void sequence_rows(const int32_t* cu, int b, int total, int& first, int& count) {
  const int lo = min(max(cu[b], 0), total), hi = min(max(cu[b + 1], 0), total);
  first = lo;
  count = max(hi - lo, 0);
}

// The sequence and the place in it of row tile `tile`, tiles counted over the
// sequences in order; false behind the last.  Every lane of a wave calls it.
__device__ __forceinline__ bool find_tile(const PrefillArgs& a, int tile_rows, int64_t tile, int& b, int& local,
                                          int& n_tiles) {
  const int lane = threadIdx.x & 63;
  int64_t before = 0;
  for (int base = 0; base < a.B; base += 64) {
    int first, count = 0;
    if (base + lane < a.B) sequence_rows(a.cu_q, base + lane, a.T_q, first, count);
    const int n = (int)(((int64_t)count * a.group + tile_rows - 1) / tile_rows);
    int64_t incl = n;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int64_t y = __shfl_up(incl, d, 64);
      if (lane >= d) incl += y;
    }
    const uint64_t past = __ballot(before + incl > tile);
    if (past) {
      const int w = __ffsll((unsigned long long)past) - 1;
      b = base + w;
      n_tiles = __shfl(n, w, 64);
      local = (int)(tile - before - (__shfl(incl, w, 64) - n_tiles));
      return true;
    }
    before += __shfl(incl, 63, 64);
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

constexpr int kStages = 3;  // tiles of keys and values in LDS

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
__device__ __forceinline__ void stage(const uint16_t* base, int64_t stride, int t0, int last, uint32_t lds) {
  constexpr int kCalls = kKeys * D * 2 / 1024 / WAVES, kRows = 1024 / (D * 2);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < kCalls; ++i) {
    const int call = wave * kCalls + i;
    const int row = call * kRows + lane / (D / 8);
    const int c = (staged<D>(row, lane % (D / 8)) % (D * 2)) / 16;
    async_load_1k(base + (int64_t)min(t0 + row, last) * stride + 8 * c, lds + 1024 * call);
  }
}

template <int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void attn_prefill_kernel(PrefillArgs a) {
  constexpr int kTileRows = kWaveRows * WAVES, kTileBytes = kKeys * D * 2;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kStages][2][kTileBytes];

  int b, local, n_tiles;
  if (!find_tile(a, kTileRows, blockIdx.x, b, local, n_tiles)) return;
  local = n_tiles - 1 - local;  // a sequence's longest rows first
  int q0, lq, k0, lk;
  sequence_rows(a.cu_q, b, a.T_q, q0, lq);
  sequence_rows(a.cu_k, b, a.T_k, k0, lk);
  if (a.status && blockIdx.y == 0 && threadIdx.x == 0 &&
      (q0 != a.cu_q[b] || q0 + lq != a.cu_q[b + 1] || k0 != a.cu_k[b] || k0 + lk != a.cu_k[b + 1]))
    atomicOr(a.status, MOE_DEV_BAD_LENGTH);

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 31, h = lane >> 5;
  const int kvh = blockIdx.y;
  const int64_t n_rows = (int64_t)lq * a.group;
  const int64_t row0 = (int64_t)local * kTileRows;
  const int64_t r = row0 + wave * kWaveRows + col;
  const bool live = r < n_rows;
  const int64_t rc = live ? r : n_rows - 1;
  const int tok = (int)(rc / a.group), head = kvh * a.group + (int)(rc - (int64_t)tok * a.group);
  // the last key that this row sees, that the tile's first row sees and that its last row sees
  const int limit = min(a.causal ? tok + lk - lq : lk - 1, lk - 1);
  const int first_limit = min(a.causal ? (int)(row0 / a.group) + lk - lq : lk - 1, lk - 1);
  const int tile_last = a.causal ? (int)((min(row0 + kTileRows, n_rows) - 1) / a.group) + lk - lq : lk - 1;
  const int n_key_tiles = tile_last < 0 ? 0 : tile_last / kKeys + 1;

  v16f o[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) o[i] = v16f{};
  float m = kNoScore, l = 0.0f;

  if (n_key_tiles > 0) {
    v8bf qf[D / 16];
    const uint16_t* qrow = a.q + (q0 + (int64_t)tok) * a.q_stride + head * D + 8 * h;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) qf[i] = *reinterpret_cast<const v8bf*>(qrow + 16 * i);

    const uint16_t* kbase = a.k + (int64_t)k0 * a.k_stride + kvh * D;
    const uint16_t* vbase = a.v + (int64_t)k0 * a.v_stride + kvh * D;
    const uint32_t lds0 = lds_address(lds);
    const auto fetch = [&](int kt, int st) {
      stage<D, WAVES>(kbase, a.k_stride, kt * kKeys, lk - 1, lds0 + (2 * st) * kTileBytes);
      stage<D, WAVES>(vbase, a.v_stride, kt * kKeys, lk - 1, lds0 + (2 * st + 1) * kTileBytes);
    };
    const auto scores = [&](const uint8_t* lds_k, v16f (&s)[2]) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        s[u] = v16f{};
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
          const v8bf kf = *reinterpret_cast<const v8bf*>(lds_k + staged<D>(32 * u + col, 2 * i + h));
          s[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[i], s[u], 0, 0, 0);
        }
      }
    };

    fetch(0, 0);
    wait_async_and_barrier<0>();
    if (n_key_tiles > 1) fetch(1, 1);
    v16f s[2], s_next[2];
    scores(lds[0][0], s);
    int st = 0;
    for (int kt = 0; kt < n_key_tiles; ++kt) {
      const int st1 = st == kStages - 1 ? 0 : st + 1, st2 = st1 == kStages - 1 ? 0 : st1 + 1;
      // tile kt + 1 is here, and every wave is done with tile kt - 1, whose place tile kt + 2 takes
      wait_async_and_barrier<0>();
      if (kt + 2 < n_key_tiles) fetch(kt + 2, st2);
      // the next tile's scores: matrix work beside this tile's softmax.  Behind the last tile they are not used.
      scores(lds[st1][0], s_next);

      const int t0 = kt * kKeys;
      if (t0 + kKeys - 1 > first_limit) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (t0 + 32 * u + 8 * (i / 4) + 4 * h + (i & 3) > limit) s[u][i] = -INFINITY;
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
        l *= alpha;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) o[i] *= alpha;
      }
      float sum = 0.0f;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[u][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][i], a.c, -m));
          sum += s[u][i];
        }
      l += sum;

      const uint8_t* lds_v = lds[st][1];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          union {
            v8bf v;
            uint32_t x[4];
          } p;
#pragma unroll
          for (int i = 0; i < 4; ++i) p.x[i] = pack_bf16(s[u][8 * w + 2 * i], s[u][8 * w + 2 * i + 1]);
          // lane j of a 16-lane group gives the address of row j / 4, 8-byte piece j % 4 of a 4 x 16 block and
          // gets column j of it
          const int row = 32 * u + 16 * w + 4 * h + ((lane & 15) >> 2);
#pragma unroll
          for (int dt = 0; dt < D / 32; ++dt) {
            const int c = 4 * dt + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), piece = 8 * (lane & 1);
            union {
              v8bf v;
              v4s x[2];
            } vf;
            vf.x[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) v4s*)(lds_v + staged<D>(row, c) + piece));
            vf.x[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) v4s*)(lds_v + staged<D>(row + 8, c) + piece));
            o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf.v, p.v, o[dt], 0, 0, 0);
          }
        }
#pragma unroll
      for (int u = 0; u < 2; ++u) s[u] = s_next[u];
      st = st1;
    }
  }

  l += __shfl_xor(l, 32, 64);
  if (!live) return;
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
  uint16_t* orow = a.out + ((q0 + (int64_t)tok) * (a.kv_heads * a.group) + head) * D + 4 * h;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<uint2*>(orow + 32 * dt + 8 * i) =
          make_uint2(pack_bf16(o[dt][4 * i] * inv, o[dt][4 * i + 1] * inv),
                     pack_bf16(o[dt][4 * i + 2] * inv, o[dt][4 * i + 3] * inv));
}

template <int D>
moe_status_t launch_prefill(const PrefillArgs& a, hipStream_t stream) {
  constexpr int kWaves = 8;
  const int64_t tiles = (int64_t)a.T_q * a.group / (kWaves * kWaveRows) + a.B;  // sequences may each add a part of one
  if (tiles * kWaves * 64 >= (int64_t)1 << 32)
    return fail(MOE_ERR_UNSUPPORTED_SHAPE, "moe_attn_prefill: %lld row tiles", (long long)tiles);
  MOE_LAUNCH("attn_prefill", (attn_prefill_kernel<D, kWaves>), dim3((unsigned)tiles, a.kv_heads), dim3(64 * kWaves), 0,
             stream, a);
  return check_launch("moe_attn_prefill");
}

}  // namespace

}  // namespace moe

using namespace moe;

extern "C" size_t moe_attn_prefill_workspace(moe_attn_dims_t d, int32_t B, int32_t T_q, int32_t max_k) {
  (void)d;
  (void)B;
  (void)T_q;
  (void)max_k;
  return 0;
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
  if (B == 0 || T_q == 0) return MOE_OK;
  if ((st = check_rows(q, q_stride, d.q_heads, d.head_dim, "moe_attn_prefill", "q")) != MOE_OK) return st;
  if (T_k > 0 && (st = check_rows(k, k_stride, d.kv_heads, d.head_dim, "moe_attn_prefill", "k")) != MOE_OK) return st;
  if (T_k > 0 && (st = check_rows(v, v_stride, d.kv_heads, d.head_dim, "moe_attn_prefill", "v")) != MOE_OK) return st;
  if (!cu_q || !cu_k || !out) return fail(MOE_ERR_INVALID_ARG, "moe_attn_prefill: null pointer");
  if (!aligned(out, 16)) return fail(MOE_ERR_INVALID_ARG, "moe_attn_prefill: out must be 16-byte aligned");
  const size_t need = moe_attn_prefill_workspace(d, B, T_q, max_k);
  if (need && (!ws || ws_bytes < need || !aligned(ws, 256)))
    return fail(MOE_ERR_WORKSPACE, "moe_attn_prefill: workspace %zu bytes, needs %zu, 256-byte aligned", ws_bytes, need);
  const PrefillArgs a{q, k, v, q_stride, k_stride, v_stride, cu_q, cu_k, out, dev_status,
                      B, T_q, T_k, d.kv_heads, d.q_heads / d.kv_heads, causal != 0, scale * kLog2e};
  return d.head_dim == 64 ? launch_prefill<64>(a, stream) : launch_prefill<128>(a, stream);
}
