// Products of up to 16 rows a matrix with 4-bit weights: every weight is read once
// and the kernel is bound by that stream.  (64 tokens of Zipf routing, gate/up of 256
// experts of 7168 x 2048: 2.2 GB in 358 us, 6.1 TB/s, where a plain read reaches 7.0; down:
// 1.1 GB in 210 us.  One token, gate/up: 125 MB in 24.9 us, 8 of them for the launch, the
// sort and the first weights' way, then 7.4 TB/s.  One row by 16384 x 7168: 62 MB in 13.0 us.)
//
// An item is R tiles of 16 weight rows, 2 or 1 (with GATEUP half of them W_gate's and half
// the same rows of W_up) against a tile of up to 16 activation rows.  A workgroup
// takes a run of neighbouring items, so neighbouring weights and mostly the same
// activations: wave w keeps the activations' K blocks of 128 from NBW w to
// NBW w + NBW - 1 in registers from one item to the next and streams those blocks
// of the weights; the waves' sums are added through LDS in wave order.  So the loop
// over items loads weights and scales alone.  D items are in flight: a register is
// loaded again, for the item D further on, as soon as it has been used.  (With a workgroup
// an item, which loads its activations, that one token's layer took 72.6 us, so 53.0.)
// NBW is 1, 2, 4 or 8: a line of 128 bytes of scales that one wave asks for while another's load
// has it on its way stalls both, and with these no line is two waves' (3 and 5 blocks a wave, which
// would leave no wave without work, took 42.2 us for the layer against 40.4).
//
// The matrix instruction is 16x16x32 bf16 with the weights as its first operand:
// 32 columns are one scale group, expanded to bf16 with the scale in it, and a
// result register holds four neighbouring outputs of one activation row.
#include <algorithm>

#include "w4.h"
#include "w4_rows.h"

namespace moe {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Waves of a CU, so that NBW blocks of activations fit their registers.
constexpr int few_waves(int nbw) { return nbw <= 2 ? 16 : nbw <= 4 ? 12 : 8; }
constexpr int kFewMaxWaves = 8;    // of a workgroup
constexpr int kFewMaxBlocks = 64;  // K blocks: 8 waves of 8
// Row tiles of experts: at most one an expert, and one for 16 rows.
constexpr int few_tiles(int rows, int E) { return (rows < E ? rows : E) + rows / 16; }

enum FewMode { kDense, kExperts, kExpertsGateUp, kSlotsGateUp };

template <int NBW, int R, int D, FewMode MODE>
__global__ __launch_bounds__(64 * kFewMaxWaves, few_waves(NBW) / 4) void w4_few_kernel(W4Args p, int rows, W4Slots slots) {
  constexpr bool GATEUP = MODE == kExpertsGateUp || MODE == kSlotsGateUp;
  constexpr int kTiles = GATEUP ? R / 2 : R;  // tiles of outputs
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int waves = blockDim.x >> 6;
  v4f* red = reinterpret_cast<v4f*>(lds);  // [2][waves][R][64]
  const int r = lane & 15, kq = lane >> 4;
  const int nb = p.K / kBlock;
  const int groups = p.N / 16;
  const int items_n = (groups + kTiles - 1) / kTiles;
  const W4Range range = w4_part(p, blockIdx.y, 4);  // whole pieces of the scales' layout
  const int kb0 = range.b0 + wave * NBW, last = range.b0 + range.n - 1;
  const int64_t chunks = (nb + 3) / 4;

  // The row tiles, and this workgroup's items: neighbouring ones, of neighbouring weights.
  int m_tiles = (rows + 15) / 16;
  int2* list = reinterpret_cast<int2*>(lds + (size_t)2 * waves * R * 1024);
  int* slot_src = reinterpret_cast<int*>(list + kSortSlots);  // kSlotsGateUp
  // What the launch behind this one, and the caller, need to know of the slots.
  auto report_slots = [&]() {
    const int bad = slot_errors(slots.ids, rows, p.topk, p.E);
    if (slots.dev_status && bad && lane == 0) atomicOr(slots.dev_status, bad);
    if (lane == 0) slots.list[kSortSlots] = make_int2(m_tiles, 0);
  };
  // One token's slots need no sort: slot j is row tile j (one with a bad id is computed with expert 0, which
  // nothing but this token's output sees).
  const bool one = MODE == kSlotsGateUp && rows == p.topk;
  if (one) {
    m_tiles = rows;
  } else if constexpr (MODE == kSlotsGateUp) {
    int* count = slot_src + kSortSlots;
    if (wave == 0) {
      int place;
      const int n = sort_slots(slots.ids, rows, p.E, list, slot_src, place);
      if (lane == 0) *count = n;
      if (blockIdx.x == 0 && lane < rows) slots.dest_row[lane] = place;
    }
    __syncthreads();
    m_tiles = __builtin_amdgcn_readfirstlane(*count);
    if (blockIdx.x == 0 && wave == waves - 1) {  // also where no slot has an expert
      report_slots();
      if (lane < m_tiles) slots.list[lane] = list[lane];
    }
  } else if constexpr (MODE != kDense) {
    const int most = few_tiles(rows, p.E);
    if (wave == 0) {
      const int n = list_row_tiles(p.offsets, p.E, 16, rows, most, list);
      if (lane == 0) list[most] = make_int2(n, 0);
    }
    __syncthreads();
    m_tiles = __builtin_amdgcn_readfirstlane(list[most].x);
  }
  // (A division of 64 bits is a hundred instructions: the launch sees to it that the items fit 32.)
  const uint32_t items = (uint32_t)(m_tiles * items_n);
  const uint32_t each = items / gridDim.x, more = items - each * gridDim.x;  // the first `more` workgroups take one more
  const uint32_t first = blockIdx.x * each + min(blockIdx.x, more);
  int todo = (int)(each + (blockIdx.x < more ? 1u : 0u));
  if (todo == 0) return;

  struct Tile {
    int a, e, p0, m;
  };
  auto find = [&](int a) {
    if constexpr (MODE == kDense) return Tile{a, 0, a * 16, min(16, rows - a * 16)};
    if (one) {
      const int e = slots.ids[a];
      return Tile{a, (uint32_t)e < (uint32_t)p.E ? e : 0, a, 1};
    }
    const int p0 = __builtin_amdgcn_readfirstlane(list[a].x), em = __builtin_amdgcn_readfirstlane(list[a].y);
    return Tile{a, em & 0xffff, p0, em >> 16};
  };

  // What is loaded next: item lg of row tile lk.
  Tile lk = find((int)(first / (uint32_t)items_n));
  int lg = (int)(first - (uint32_t)lk.a * items_n);
  int left = todo;  // items that are not loaded yet
  const uint8_t *w_base[GATEUP ? 2 : 1], *s_base[GATEUP ? 2 : 1];
  auto point = [&]() {
    const int64_t g = (int64_t)lk.e * groups;
    w_base[0] = p.w0 + g * nb * kW4TileBytes;
    s_base[0] = p.s0 + g * chunks * kW4ScaleTile;
    if constexpr (GATEUP) {
      w_base[1] = p.w1 + g * nb * kW4TileBytes;
      s_base[1] = p.s1 + g * chunks * kW4ScaleTile;
    }
  };
  point();
  struct Codes {
    u32x4 w[R][NBW];
    uint32_t s[R][NBW];
  };
  auto load = [&](Codes& q, int t) {  // tile t of the item
    const int mat = GATEUP && t >= kTiles ? 1 : 0;
    const int64_t g = min(lg * kTiles + (GATEUP ? t % kTiles : t), groups - 1);
    const uint8_t* w = w_base[mat] + g * nb * kW4TileBytes;
#pragma unroll
    for (int u = 0; u < NBW; ++u)  // blocks past the last are that one again, against zeros
      q.w[t][u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(w + min(kb0 + u, last) * kW4TileBytes + lane * 16));
    const uint8_t* s = s_base[mat] + g * chunks * kW4ScaleTile + r * 16;
    // (behind the last column's scales there is padding to be read, and a wave without blocks reads the last ones)
    const int sb = min(kb0, last) & ~(NBW - 1);
    s += (sb >> 2) * kW4ScaleTile + (sb & 3) * 4;
    if constexpr (NBW >= 4) {
#pragma unroll
      for (int c = 0; c < NBW / 4; ++c) {
        const u32x4 v = *reinterpret_cast<const u32x4*>(s + (c ? min(c, (last >> 2) - (sb >> 2)) : 0) * kW4ScaleTile);
#pragma unroll
        for (int u = 0; u < 4; ++u) q.s[t][4 * c + u] = v[u];
      }
    } else if constexpr (NBW == 2) {
      const u32x2 v = *reinterpret_cast<const u32x2*>(s);
      q.s[t][0] = v[0];
      q.s[t][1] = v[1];
    } else {
      q.s[t][0] = *reinterpret_cast<const uint32_t*>(s);
    }
  };
  // (An expert's items are at least D, so the item that is multiplied next is of this row tile or the one before.)
  auto next_item = [&]() {
    if (--left <= 0) return;  // the last item is loaded again, and not used
    if (++lg < items_n) return;
    lg = 0;
    lk = find(lk.a + 1);
    point();
  };

  Codes q[D];
  Tile ck = lk;
  int cg = lg;
  w4_bf16x8 x[NBW][4];
  auto load_x = [&]() {
    // Lanes without an activation row load nothing: the address path takes as long for a row that sixteen lanes share.
    int64_t row = ck.p0 + min(r, ck.m - 1);
    if constexpr (MODE == kSlotsGateUp) {
      row = one ? 0 : slot_src[row] / p.topk;
    } else if (p.sorted_src) {
      row = p.sorted_src[row] / p.topk;
      if (row < 0 || row >= p.x_rows) row = 0;
    }
    const uint16_t* xr = p.x + row * p.x_stride + 8 * kq;
#pragma unroll
    for (int u = 0; u < NBW; ++u)
#pragma unroll
      for (int j = 0; j < 4; ++j) x[u][j] = __builtin_bit_cast(w4_bf16x8, make_uint4(0, 0, 0, 0));
    if (r < ck.m) {
#pragma unroll
      for (int u = 0; u < NBW; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          x[u][j] = __builtin_bit_cast(w4_bf16x8, *reinterpret_cast<const uint4*>(xr + min(kb0 + u, last) * kBlock + 32 * j));
    }
    if (kb0 + NBW - 1 > last) {  // the last wave
#pragma unroll
      for (int u = 0; u < NBW; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          x[u][j] = kb0 + u <= last ? x[u][j] : __builtin_bit_cast(w4_bf16x8, make_uint4(0, 0, 0, 0));
    }
  };
#pragma unroll
  for (int d = 0; d < D; ++d) {
    if (d) next_item();
#pragma unroll
    for (int t = 0; t < R; ++t) load(q[d], t);
  }
  load_x();
  if (one && blockIdx.x == 0 && wave == waves - 1) {
    report_slots();
    if (lane < rows) {
      const int e = slots.ids[lane];
      slots.list[lane] = make_int2(lane, ((uint32_t)e < (uint32_t)p.E ? e : 0) | 1 << 16);
      slots.dest_row[lane] = lane;
    }
  }

  int parity = 0;
  auto item = [&](Codes& c) {
    next_item();
    v4f* mine = red + parity * waves * R * 64;
#pragma unroll
    for (int t = 0; t < R; ++t) {
      v4f acc = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int u = 0; u < NBW; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w4_expand(c.w[t][u][j], w4_scale(c.s[t][u], j)), x[u][j], acc, 0, 0, 0);
      load(c, t);
      mine[(wave * R + t) * 64 + lane] = acc;
    }
    // A plain barrier: loads stay in flight across it.
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    // The waves' sums, in wave order.  Other waves finish the next item's, and all go on meanwhile.
    for (int t = (wave + waves - cg * kTiles % waves) % waves; t < kTiles; t += waves) {
      v4f v = mine[t * 64 + lane];
      for (int w = 1; w < waves; ++w) v += mine[(w * R + t) * 64 + lane];
      if (GATEUP) {
        v4f u = mine[(kTiles + t) * 64 + lane];
        for (int w = 1; w < waves; ++w) u += mine[(w * R + kTiles + t) * 64 + lane];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = silu_mul(v[i], u[i]);
      }
      if (r < ck.m && cg * kTiles + t < groups) w4_store(p, (int64_t)ck.p0 + r, (cg * kTiles + t) * 16 + 4 * kq, v);
    }
    parity ^= 1;
    --todo;
    if (++cg == items_n && todo > 0) {
      cg = 0;
      ck = lk;
      load_x();
    }
  };
  static_assert(D == 1 || D == 2 || D == 4, "the loop below is written out");
  while (true) {
    item(q[0]);
    if (todo == 0) return;
    if constexpr (D > 1) {
      item(q[1]);
      if (todo == 0) return;
    }
    if constexpr (D > 2) {
      item(q[2]);
      if (todo == 0) return;
      item(q[3]);
      if (todo == 0) return;
    }
  }
}

// K blocks of a workgroup: a part's, whole groups of four.
int few_blocks(const W4Args& a) {
  const int splits = std::max(1, a.splits), nb = a.K / kBlock;
  return splits == 1 ? nb : 4 * (((nb + 3) / 4 + splits - 1) / splits);
}

template <int NBW, int D, FewMode MODE, int R = 2>
moe_status_t launch_few(const W4Args& a, int rows, const W4Slots& slots, hipStream_t stream) {
  constexpr bool kGateUp = MODE == kExpertsGateUp || MODE == kSlotsGateUp;
  const char* name = kGateUp ? "w4_few_gateup" : "w4_few";
  const int splits = std::max(1, a.splits);
  const int waves = (few_blocks(a) + NBW - 1) / NBW;
  const int tiles = kGateUp ? R / 2 : R;
  const int64_t items_n = (a.N / 16 + tiles - 1) / tiles;
  const int64_t m_tiles = MODE == kDense ? (rows + 15) / 16 : few_tiles(rows, a.E);
  if (items_n * m_tiles > INT32_MAX) return fail(MOE_ERR_UNSUPPORTED_SHAPE, "%s: too many rows and columns", name);
  const int64_t blocks = std::min<int64_t>(items_n * m_tiles, std::max(1, 256 * (few_waves(NBW) / waves) / splits));
  const size_t lds = (size_t)2 * waves * R * 1024 + (MODE == kDense         ? 0
                                                     : MODE == kSlotsGateUp ? kSortSlots * sizeof(int2) + (kSortSlots + 1) * sizeof(int)
                                                                            : (m_tiles + 1) * sizeof(int2));
  MOE_LAUNCH(name, (w4_few_kernel<NBW, R, D, MODE>), dim3((unsigned)blocks, splits), dim3(64 * waves), lds, stream, a, rows, slots);
  return check_launch(name);
}

// NBW: a wave's K blocks.
template <FewMode MODE>
moe_status_t few_by_length(const W4Args& a, int rows, const W4Slots& slots, hipStream_t stream) {
  const int nb = few_blocks(a);
  if constexpr (MODE == kDense) {
    // Items of one tile where items of two leave half of the CUs without work (1, 16 rows by 7168 x 4096: 8.0, 11.6 against 8.9,
    // 13.2 us; 4096 x 2048: 5.1, 7.1 against 5.6, 8.2; 192 items of two, 2048 x 6144: 5.1, 7.2 against 4.4, 5.6).
    if (nb > 8 && (int64_t)a.N / 32 * std::max(1, a.splits) <= 128) {
      if (nb <= 32) return launch_few<4, 1, MODE, 1>(a, rows, slots, stream);
      return launch_few<8, 1, MODE, 1>(a, rows, slots, stream);
    }
  }
  if (nb <= 4) return launch_few<1, 4, MODE>(a, rows, slots, stream);
  if (nb <= 8) return launch_few<2, 2, MODE>(a, rows, slots, stream);
  if (nb <= 32) return launch_few<4, 1, MODE>(a, rows, slots, stream);
  return launch_few<8, 1, MODE>(a, rows, slots, stream);
}

}  // namespace

bool w4_few_fits(int32_t K) { return K / kBlock <= kFewMaxBlocks; }

// Parts of K of one matrix whose rows are longer than a workgroup holds.
int w4_few_parts(int32_t K) { return w4_few_fits(K) ? 1 : (K / kBlock + 31) / 32; }

// Experts: at most kFewMaxRows rows.
moe_status_t run_w4_few(const W4Args& a, bool gateup, int64_t rows, hipStream_t stream) {
  if (!a.offsets) return few_by_length<kDense>(a, (int)rows, W4Slots{}, stream);
  return gateup ? few_by_length<kExpertsGateUp>(a, (int)rows, W4Slots{}, stream)
                : few_by_length<kExperts>(a, (int)rows, W4Slots{}, stream);
}

// Gate and up of at most kSortSlots slots that nothing has sorted yet.
moe_status_t run_w4_few_slots(const W4Args& a, int rows, const W4Slots& slots, hipStream_t stream) {
  return few_by_length<kSlotsGateUp>(a, rows, slots, stream);
}

}  // namespace moe
