// Products of a few rows with 4-bit weights: every weight is read once and the
// kernel is bound by that stream.
//
// An item is R tiles of 16 weight rows (with GATEUP one of W_gate and the same one
// of W_up) against a tile of up to 16 MT activation rows.  A workgroup takes a run of
// neighbouring items; its W waves take contiguous parts of K of each and their sums
// are added through LDS in wave order.
// The matrix instruction is 16x16x32 bf16 with the weights as its first operand:
// 32 columns are one scale group, expanded to bf16 with the scale in it, and a
// result register holds four neighbouring outputs of one activation row.
//
// A wave has the codes of U K blocks of 128 in flight while it multiplies U others,
// the next item's among them when an item ends.
#include <algorithm>

#include "w4.h"
#include "w4_rows.h"

namespace moe {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <int MT, int R, int W, int U, bool GATEUP>
__global__ __launch_bounds__(64 * W, MT == 4 ? 2 : 4) void w4_gemv_kernel(W4Args p, int64_t rows) {
  static_assert(!GATEUP || R == 2, "one tile of each projection");
  constexpr int kTiles = GATEUP ? 1 : R;  // tiles of outputs
  __shared__ v4f red[2][W][R * MT][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, kq = lane >> 4;
  const int nb = p.K / kBlock;
  const int groups = p.N / 16;
  const int items_n = (groups + kTiles - 1) / kTiles;
  const int kb0 = (int)((int64_t)wave * nb / W), kb1 = (int)((int64_t)(wave + 1) * nb / W);
  const int turns = ((nb + W - 1) / W + U - 1) / U;  // of every wave: the one with the most blocks decides
  const int64_t chunks = (nb + 3) / 4;

  // This workgroup's items: neighbouring ones, of neighbouring weights.
  const int64_t m_tiles = p.offsets ? all_tiles(p.offsets, p.E, 16 * MT, (int)rows) : (rows + 16 * MT - 1) / (16 * MT);
  const int64_t items = m_tiles * items_n;
  const int64_t first = items * blockIdx.x / gridDim.x, end = items * (blockIdx.x + 1) / gridDim.x;
  if (first >= end) return;

  struct Tile {
    int64_t a;
    int e, m;
    int64_t p0;
  };
  auto find = [&](int64_t a) {
    if (!p.offsets) return Tile{a, 0, (int)min((int64_t)16 * MT, rows - a * 16 * MT), a * 16 * MT};
    const ExpertRows t = find_row_tile(p.offsets, p.E, (int)a, 16 * MT, (int)rows);
    return Tile{a, t.e, t.m, t.p0};
  };

  struct Blocks {
    u32x4 w[U][R];
    uint32_t s[U][R];
  };
  // What is loaded next: turn `lt` of item (lk, lg), whose weights begin at wt and st.
  Tile lk = find(first / items_n);
  int lg = (int)(first - lk.a * items_n), lt = 0;
  int64_t left = (end - first) * turns;  // turns that are not loaded yet
  const uint8_t *wt[R], *st[R];
  auto point = [&]() {
#pragma unroll
    for (int t = 0; t < R; ++t) {
      const bool second = GATEUP && t == 1;
      const int64_t g = (int64_t)lk.e * groups + (GATEUP ? lg : min(lg * R + t, groups - 1));
      wt[t] = (second ? p.w1 : p.w0) + g * nb * kW4TileBytes + lane * 16;
      st[t] = (second ? p.s1 : p.s0) + g * chunks * kW4ScaleTile + r * 16;
    }
  };
  point();
  auto load = [&](Blocks& q) {  // blocks past the wave's last are that one again
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = max(min(kb0 + lt * U + u, kb1 - 1), 0);
#pragma unroll
      for (int t = 0; t < R; ++t) {
        q.w[u][t] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(wt[t] + (int64_t)c * kW4TileBytes));
        q.s[u][t] = *reinterpret_cast<const uint32_t*>(st[t] + (c >> 2) * kW4ScaleTile + (c & 3) * 4);
      }
    }
    if (--left <= 0) return;  // the last turn is loaded again, and not used
    if (++lt < turns) return;
    lt = 0;
    if (++lg == items_n) {
      lg = 0;
      lk = find(lk.a + 1);
    }
    point();
  };

  // What is multiplied: turn `ct` of item (ck, cg).
  Blocks q0, q1;
  Tile ck = lk;
  int cg = lg, ct = 0, parity = 0;
  load(q0);
  // Rows past the last read that one again: what a lane has for an activation row reaches that row's sums alone, which
  // are not stored.
  const uint16_t* xr[MT];
  auto point_x = [&]() {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      int64_t row = ck.p0 + min(mt * 16 + r, ck.m - 1);
      if (p.sorted_src) {
        row = p.sorted_src[row] / p.topk;
        if (row < 0 || row >= p.x_rows) row = 0;
      }
      xr[mt] = p.x + row * p.x_stride + 8 * kq;
    }
  };
  point_x();
  v4f acc[R][MT];
  auto clear = [&]() {
#pragma unroll
    for (int t = 0; t < R; ++t)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) acc[t][mt] = v4f{0.f, 0.f, 0.f, 0.f};
  };
  clear();

  auto turn = [&](const Blocks& q, Blocks& next) {
    const int b = kb0 + ct * U;
    // Loads come back in order: a turn's activations go out in front of the next turn's weights, or their wait
    // would be for those too.
    w4_bf16x8 x[U][MT][4];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          x[u][mt][j] = __builtin_bit_cast(w4_bf16x8, *reinterpret_cast<const uint4*>(
                                                          xr[mt] + (int64_t)max(min(b + u, kb1 - 1), 0) * kBlock + 32 * j));
    __builtin_amdgcn_sched_barrier(0);
    load(next);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (b + u >= kb1) break;
#pragma unroll
      for (int t = 0; t < R; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const w4_bf16x8 w = w4_expand(q.w[u][t][j], w4_scale(q.s[u][t], j));
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
            acc[t][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x[u][mt][j], acc[t][mt], 0, 0, 0);
        }
    }
    if (++ct < turns) return;
    // The item is done: the waves' sums, in wave order.  Another wave finishes each item, while the others go on.
    ct = 0;
#pragma unroll
    for (int t = 0; t < R; ++t)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) red[parity][wave][t * MT + mt][lane] = acc[t][mt];
    // (a plain barrier: loads stay in flight across it)
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    for (int i = (wave + cg) % W; i < kTiles * MT; i += W) {
      const int t = i / MT, mt = i % MT;
      v4f v = red[parity][0][i][lane];
#pragma unroll
      for (int w = 1; w < W; ++w) v += red[parity][w][i][lane];
      if (GATEUP) {
        v4f u = red[parity][0][MT + i][lane];
#pragma unroll
        for (int w = 1; w < W; ++w) u += red[parity][w][MT + i][lane];
#pragma unroll
        for (int c = 0; c < 4; ++c) v[c] = silu_mul(v[c], u[c]);
      }
      if (mt * 16 + r < ck.m && cg * kTiles + t < groups) w4_store(p, ck.p0 + mt * 16 + r, (cg * kTiles + t) * 16 + 4 * kq, v);
    }
    parity ^= 1;
    clear();
    if (++cg == items_n) {
      cg = 0;
      if (ck.a + 1 < m_tiles) {
        ck = find(ck.a + 1);
        point_x();
      }
    }
  };
  for (int64_t n = (end - first) * turns; n > 0; n -= 2) {
    turn(q0, q1);
    if (n == 1) break;
    turn(q1, q0);
  }
}

template <int MT, int R, int W, int U, bool GATEUP>
moe_status_t launch_gemv(const W4Args& a, int64_t rows, hipStream_t stream) {
  const char* name = GATEUP ? "w4_gemv_gateup" : "w4_gemv";
  const int tiles = GATEUP ? 1 : R;
  const int64_t items_n = (a.N / 16 + tiles - 1) / tiles;
  // Row tiles of experts: each may leave its last one unfilled.
  const int64_t m_tiles = a.offsets ? rows / (16 * MT) + (rows < a.E ? rows : (int64_t)a.E) : (rows + 16 * MT - 1) / (16 * MT);
  const int64_t blocks = std::min<int64_t>(items_n * m_tiles, 256 * 16 / W);
  MOE_LAUNCH(name, (w4_gemv_kernel<MT, R, W, U, GATEUP>), dim3((unsigned)blocks), dim3(64 * W), 0, stream, a, rows);
  return check_launch(name);
}

}  // namespace

moe_status_t run_w4_gemv(const W4Args& a, bool gateup, int64_t rows, hipStream_t stream) {
  if (gateup) return launch_gemv<1, 2, 8, 2, true>(a, rows, stream);
  if (a.offsets || rows <= 16) return launch_gemv<1, 2, 8, 2, false>(a, rows, stream);
  if (rows <= 32) return launch_gemv<2, 2, 8, 1, false>(a, rows, stream);
  return launch_gemv<4, 2, 4, 1, false>(a, rows, stream);
}

}  // namespace moe
