// Products of a few rows with 4-bit weights: every weight is read once and the
// kernel is bound by that stream.
//
// A workgroup takes R tiles of 16 weight rows (with GATEUP one of W_gate and the
// same one of W_up) against up to 16 MT activation rows; its W waves take
// contiguous parts of K and their sums are added through LDS in wave order.
// The matrix instruction is 16x16x32 bf16 with the weights as its first operand:
// 32 columns are one scale group, expanded to bf16 with the scale in it, and a
// result register holds four neighbouring outputs of one activation row.
//
// A wave has four K blocks of 128 in flight while it multiplies four others.
#include "w4.h"
#include "w4_rows.h"

namespace moe {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kGemvBlocks = 4;  // K blocks that a wave loads together

template <int MT, int R, int W, bool GATEUP>
__global__ __launch_bounds__(64 * W) void w4_gemv_kernel(W4Args p, int m_lo, int m_hi, int64_t rows) {
  static_assert(!GATEUP || R == 2, "one tile of each projection");
  constexpr int kTiles = GATEUP ? 1 : R;  // tiles of outputs
  __shared__ v4f red[W][R * MT][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, kq = lane >> 4;
  const int nb = p.K / kBlock;
  const int groups = p.N / 16;
  const int items_n = (groups + kTiles - 1) / kTiles;
  const int kb0 = (int)((int64_t)wave * nb / W), kb1 = (int)((int64_t)(wave + 1) * nb / W);

  int e = 0;
  int64_t p0 = 0, m_first = 0, m_end = 0;
  const int64_t a = blockIdx.x / items_n;
  const int g0 = (int)(blockIdx.x % items_n) * kTiles;
  if (p.offsets) {
    const ExpertRows ref = find_expert(p.offsets, p.E, (int)a, m_lo, m_hi, (int)rows);
    if (ref.e < 0) return;  // the whole workgroup
    e = ref.e;
    p0 = ref.p0;
    m_end = ref.m;
  } else {
    m_first = a * 16 * MT;
    m_end = min(m_first + 16 * MT, rows);
  }

  const uint8_t *wt[R], *st[R];
  const int64_t chunks = (nb + 3) / 4;
#pragma unroll
  for (int t = 0; t < R; ++t) {
    const bool second = GATEUP && t == 1;
    const int64_t g = (int64_t)e * groups + (GATEUP ? g0 : min(g0 + t, groups - 1));
    wt[t] = (second ? p.w1 : p.w0) + g * nb * kW4TileBytes + lane * 16;
    st[t] = (second ? p.s1 : p.s0) + g * chunks * kW4ScaleTile + r * 16;
  }

  struct Blocks {
    u32x4 w[kGemvBlocks][R];
    uint32_t s[kGemvBlocks][R];
  };
  auto load = [&](int b, Blocks& q) {  // blocks past the wave's last are that one again
#pragma unroll
    for (int u = 0; u < kGemvBlocks; ++u) {
      const int c = min(b + u, kb1 - 1);
#pragma unroll
      for (int t = 0; t < R; ++t) {
        q.w[u][t] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(wt[t] + (int64_t)c * kW4TileBytes));
        q.s[u][t] = *reinterpret_cast<const uint32_t*>(st[t] + (c >> 2) * kW4ScaleTile + (c & 3) * 4);
      }
    }
  };

  for (int64_t mb = m_first; mb < m_end; mb += 16 * MT) {
    const uint16_t* xr[MT];
    bool there[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const int64_t m = mb + mt * 16 + r;
      there[mt] = m < m_end;
      int64_t row = p0 + min(m, m_end - 1);
      if (p.sorted_src) {
        row = p.sorted_src[row] / p.topk;
        there[mt] = there[mt] && row >= 0 && row < p.x_rows;
      }
      xr[mt] = p.x + (there[mt] ? row : 0) * p.x_stride + 8 * kq;
    }
    v4f acc[R][MT];
#pragma unroll
    for (int t = 0; t < R; ++t)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) acc[t][mt] = v4f{0.f, 0.f, 0.f, 0.f};

    auto multiply = [&](int b, const Blocks& q) {
#pragma unroll
      for (int u = 0; u < kGemvBlocks; ++u) {
        if (b + u >= kb1) break;
        w4_bf16x8 x[MT][4];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            x[mt][j] = there[mt] ? __builtin_bit_cast(w4_bf16x8, *reinterpret_cast<const uint4*>(xr[mt] + (int64_t)(b + u) * kBlock + 32 * j))
                                 : __builtin_bit_cast(w4_bf16x8, make_uint4(0, 0, 0, 0));
#pragma unroll
        for (int t = 0; t < R; ++t)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const w4_bf16x8 w = w4_expand(q.w[u][t][j], w4_scale(q.s[u][t], j));
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
              acc[t][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x[mt][j], acc[t][mt], 0, 0, 0);
          }
      }
    };
    if (kb0 < kb1) {
      Blocks q0, q1;
      load(kb0, q0);
      for (int b = kb0; b < kb1; b += 2 * kGemvBlocks) {
        load(b + kGemvBlocks, q1);
        multiply(b, q0);
        if (b + kGemvBlocks >= kb1) break;
        load(b + 2 * kGemvBlocks, q0);
        multiply(b + kGemvBlocks, q1);
      }
    }

    // The waves' sums, in wave order; a thread finishes four outputs of one row at a time.
#pragma unroll
    for (int t = 0; t < R; ++t)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) red[wave][t * MT + mt][lane] = acc[t][mt];
    __syncthreads();
    for (int i = wave; i < kTiles * MT; i += W) {
      const int t = i / MT, mt = i % MT;
      const int64_t m = mb + mt * 16 + r;
      v4f v = red[0][i][lane];
#pragma unroll
      for (int w = 1; w < W; ++w) v += red[w][i][lane];
      if (GATEUP) {
        v4f u = red[0][MT + i][lane];
#pragma unroll
        for (int w = 1; w < W; ++w) u += red[w][MT + i][lane];
#pragma unroll
        for (int c = 0; c < 4; ++c) v[c] = silu_mul(v[c], u[c]);
      }
      if (m < m_end && g0 + t < groups) w4_store(p, p0 + m, (g0 + t) * 16 + 4 * kq, v);
    }
    __syncthreads();
  }
}

template <int MT, int R, int W, bool GATEUP>
moe_status_t launch_gemv(const W4Args& a, int64_t blocks, int m_lo, int m_hi, int64_t rows, hipStream_t stream) {
  const char* name = GATEUP ? "w4_gemv_gateup" : "w4_gemv";
  if (blocks <= 0) return MOE_OK;
  if (blocks > w4_max_blocks(64 * W)) return fail(MOE_ERR_UNSUPPORTED_SHAPE, "%s: too many rows and columns", name);
  MOE_LAUNCH(name, (w4_gemv_kernel<MT, R, W, GATEUP>), dim3((unsigned)blocks), dim3(64 * W), 0, stream, a, m_lo, m_hi, rows);
  return check_launch(name);
}

template <int R, int W, bool GATEUP>
moe_status_t launch_rows(const W4Args& a, int32_t T, int64_t rows, hipStream_t stream) {
  const int tiles = GATEUP ? 1 : R;
  const int64_t items_n = (a.N / 16 + tiles - 1) / tiles;
  if (!a.offsets) {
    if (rows <= 16) return launch_gemv<1, R, W, GATEUP>(a, items_n, 0, 0, rows, stream);
    if (rows <= 32) return launch_gemv<2, R, W, GATEUP>(a, items_n, 0, 0, rows, stream);
    return launch_gemv<4, R, W, GATEUP>(a, items_n * ((rows + 63) / 64), 0, 0, rows, stream);
  }
  // One launch for each class of experts by their rows: at most 16, 32, more (an expert has at most T rows).
  auto items = [&](int lo) { return (rows / lo < a.E ? rows / lo : (int64_t)a.E) * items_n; };
  moe_status_t st = launch_gemv<1, R, W, GATEUP>(a, items(1), 1, 16, rows, stream);
  if (st != MOE_OK || T <= 16) return st;
  st = launch_gemv<2, R, W, GATEUP>(a, items(17), 17, 32, rows, stream);
  if (st != MOE_OK || T <= 32) return st;
  return launch_gemv<4, R, W, GATEUP>(a, items(33), 33, 0x7fffffff, rows, stream);
}

}  // namespace

// `rows` activation rows in all (experts: sorted slots of T tokens).
moe_status_t run_w4_gemv(const W4Args& a, bool gateup, int32_t T, int64_t rows, hipStream_t stream) {
  if (gateup) return launch_rows<2, 4, true>(a, T, rows, stream);
  return launch_rows<2, 4, false>(a, T, rows, stream);
}

}  // namespace moe
