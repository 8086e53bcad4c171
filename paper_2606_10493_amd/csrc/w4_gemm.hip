// Products of many rows with 4-bit weights: an LDS-tiled bf16 GEMM that expands
// the weights in registers on their way from LDS to the matrix instruction.
//
// A workgroup takes a tile of up to 32 S activation rows against 256 weight rows
// (GATEUP: 128 of W_gate and the same 128 of W_up).  Its eight waves, two to a SIMD,
// share them: with H = 2 they are two halves of the activation rows by four quarters of
// the weight rows, a wave expanding 64 weight rows for up to 16 S activation rows; with
// H = 1, for small tiles, where the expansion is what counts, each has 32 weight rows
// and all activation rows, and nothing is expanded twice.  How many 16-row parts of
// activations a wave has is known when the tile is, and each number has its own loop,
// so that an expert's rows are cut into equal tiles whose size follows them.
//
// Steps of 128 K.  Activations (256 bytes a row), codes (1 KB a tile of 16 rows) and
// scales (one dword a row) go straight from global memory into LDS stages, one or
// two steps ahead, with one barrier a step; activation rows are gathered on the
// way.  The 16-byte piece c of an activation row lies at position c ^ row % 16, so
// that a quarter wave's reads fill all banks.  A step's barrier stands before the last
// quarter of the step in front of it, whose operands are in registers by then: the next
// codes are read and expanded beside those products.
#include <algorithm>
#include <type_traits>

#include "w4.h"
#include "w4_rows.h"

namespace moe {

namespace {

constexpr int kGemmWaves = 8;
constexpr int kGemmRows = 256;                         // weight rows of a workgroup
constexpr int kGemmCodes = kGemmRows / 16 * kW4TileBytes;  // of a stage
constexpr int kGemmScales = kGemmWaves * 256;          // 64 rows' for each wave
constexpr int gemm_stage(int s) { return 32 * s * 2 * kBlock + kGemmCodes + kGemmScales; }
constexpr int gemm_stages(int s) { return 3 * gemm_stage(s) <= 160 * 1024 ? 3 : 2; }

// async_load_1k's counterpart for 4 bytes a lane.
__device__ __forceinline__ void async_load_256(const void* src, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
               :
               : "s"(__builtin_amdgcn_readfirstlane((int)lds)), "v"(src)
               : "memory");
}

// The loop over K and the outputs of a wave with CNT parts of 16 activation rows and
// TILES tiles of 16 weight rows.  `load` issues the loads of a step into a stage;
// x_at, w_at and s_at are the wave's first activation part, its codes and its scales
// in stage 0.
template <int CNT, int TILES, int STAGES, int STAGE_BYTES, int LOADS, typename Load, typename Store>
__device__ __forceinline__ void w4_gemm_wave(const uint8_t* smem, int nb, int x_at, int w_at, int s_at, Load load, Store store) {
  const int lane = threadIdx.x & 63;
  const int r = lane & 15, kq = lane >> 4;
  v4f acc[TILES][CNT];
#pragma unroll
  for (int t = 0; t < TILES; ++t)
#pragma unroll
    for (int c = 0; c < CNT; ++c) acc[t][c] = v4f{0.f, 0.f, 0.f, 0.f};
  uint4 raw[TILES];
  uint32_t sc[TILES];
  auto read_codes = [&](const uint8_t* at) {
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      raw[t] = *reinterpret_cast<const uint4*>(at + w_at + t * kW4TileBytes + lane * 16);
      sc[t] = *reinterpret_cast<const uint32_t*>(at + s_at + 64 * t + 4 * r);
    }
  };
  auto expand = [&](int j, w4_bf16x8 (&w)[TILES]) {
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      const uint32_t codes = j == 0 ? raw[t].x : j == 1 ? raw[t].y : j == 2 ? raw[t].z : raw[t].w;
      w[t] = w4_expand(codes, w4_scale(sc[t], j));
    }
  };
  auto read_x = [&](const uint8_t* at, int j, int c) {
    return __builtin_bit_cast(
        w4_bf16x8, *reinterpret_cast<const uint4*>(at + x_at + (c * 16 + r) * (2 * kBlock) + (((4 * j + kq) ^ r) * 16)));
  };
#pragma unroll
  for (int s = 0; s < STAGES; ++s) load(s, s);
  wait_async_and_barrier<(STAGES - 1) * LOADS>();
  read_codes(smem);
  w4_bf16x8 w[2][TILES];
  expand(0, w[0]);
  int stage = 0;
  for (int b = 0; b < nb; ++b) {
    const uint8_t* at = smem + stage * STAGE_BYTES;
    const int next = stage + 1 == STAGES ? 0 : stage + 1;
    w4_bf16x8 x3[CNT];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (j < 3) {
#pragma unroll
        for (int c = 0; c < CNT; ++c) {
          const w4_bf16x8 x = read_x(at, j, c);
#pragma unroll
          for (int t = 0; t < TILES; ++t) acc[t][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[j & 1][t], x, acc[t][c], 0, 0, 0);
        }
        expand(j + 1, w[(j + 1) & 1]);
        if (j == 2) {
#pragma unroll
          for (int c = 0; c < CNT; ++c) x3[c] = read_x(at, 3, c);
        }
      } else {
        // Step b + 1 has landed for every wave, and every wave has read all of step b, whose stage is loaded next.
        wait_async_and_barrier<(STAGES - 2) * LOADS>();
        read_codes(smem + next * STAGE_BYTES);
        load(b + STAGES, stage);
#pragma unroll
        for (int c = 0; c < CNT; ++c)
#pragma unroll
          for (int t = 0; t < TILES; ++t) acc[t][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[1][t], x3[c], acc[t][c], 0, 0, 0);
        expand(0, w[0]);
      }
    }
    stage = next;
  }
  // No load may reach LDS after the workgroup has ended.
  wait_async_and_barrier<0>();
  // Lane 16 kq + r holds outputs 4 kq .. 4 kq + 3 of each tile for row r of each part.
#pragma unroll
  for (int c = 0; c < CNT; ++c) {
    v4f v[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) v[t] = acc[t][c];
    store(c, v);
  }
}

// Rows of one expert, or of the one matrix, are cut into the fewest tiles of at most
// 32 S rows, equal ones but for the rounding to parts of 16.
template <int S, int H, bool GATEUP>
__global__ __launch_bounds__(64 * kGemmWaves) void w4_gemm_kernel(W4Args p, int64_t rows, int n_tiles, int dealt) {
  constexpr int kXStage = 32 * S * 2 * kBlock;
  constexpr int kStage = gemm_stage(S), kStages = gemm_stages(S);
  constexpr int kXLoads = S;                      // a wave's a step: 8 S KB in all
  constexpr int kWLoads = kGemmCodes / 1024 / kGemmWaves;
  constexpr int kTiles = 2 * H;                   // 16-row weight tiles of a wave
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kStages * kStage];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = H == 2 ? wave >> 2 : 0, share = H == 2 ? wave & 3 : wave;  // of the activation rows, of the weight rows
  const int r = lane & 15, kq = lane >> 4;
  const int nb = p.K / kBlock, groups = p.N / 16;
  // Workgroups are dealt to the XCDs in turn.  Row tiles too, where there are enough of them: an XCD takes all of a row
  // tile's items one after the other, and its L2 holds the activations.
  const uint32_t x = dealt ? blockIdx.x / kXcd : blockIdx.x;
  const int turn = (int)(x / (uint32_t)n_tiles), nt = (int)(x - (uint32_t)turn * n_tiles);
  const int mt = dealt ? turn * kXcd + (int)(blockIdx.x % kXcd) : turn;
  const W4Range range = w4_part(p, blockIdx.y, 1);

  int e = 0, mc;
  int64_t p0;
  if (p.offsets) {
    const ExpertRows ref = find_even_tile(p.offsets, p.E, mt, 32 * S, (int)rows);
    if (ref.e < 0) return;  // the whole workgroup
    e = ref.e;
    p0 = ref.p0;
    mc = ref.m;
  } else {
    const int64_t tiles = (rows + 32 * S - 1) / (32 * S), part = even_tile_rows(rows, tiles);
    p0 = (int64_t)mt * part;
    if (p0 >= rows) return;
    mc = (int)min(part, rows - p0);
  }
  const int parts = (mc + 15) / 16;
  const int first = half ? (parts + 1) / 2 : 0, count = H == 1 ? parts : half ? parts / 2 : (parts + 1) / 2;

  // Sources.  Load i of the activations takes rows 32 i + 4 wave + lane / 16.
  const uint16_t* xs[kXLoads];
#pragma unroll
  for (int i = 0; i < kXLoads; ++i) {
    const int m = 32 * i + 4 * wave + (lane >> 4);
    int64_t row = p0 + min(m, mc - 1);  // rows past the tile's end read a valid one, and are not stored
    if (p.sorted_src) {
      row = p.sorted_src[row] / p.topk;
      if (row < 0 || row >= p.x_rows) row = 0;
    }
    xs[i] = p.x + row * p.x_stride + (((lane & 15) ^ (m & 15)) * 8);
  }
  // Tile t of a share: 16-row group group(t) of its matrix (groups past the last are that one again).
  auto group = [&](int t) {
    if (GATEUP) return nt * (kGemmRows / 32) + share * H + t % H;
    return nt * (kGemmRows / 16) + share * kTiles + t;
  };
  auto up = [&](int t) { return GATEUP && t >= H; };
  auto held = [&](int t) { return (int64_t)e * groups + min(group(t), groups - 1); };
  const uint8_t* ws[kWLoads];  // this wave's part of its share's tiles
#pragma unroll
  for (int i = 0; i < kWLoads; ++i) {
    const int t = half * kWLoads + i;
    ws[i] = (up(t) ? p.w1 : p.w0) + held(t) * nb * kW4TileBytes + lane * 16;
  }
  const int st = (lane >> 4) % kTiles;  // lane 16 t + r: row r of tile t
  const uint8_t* ss = (up(st) ? p.s1 : p.s0) + held(st) * ((nb + 3) / 4) * kW4ScaleTile + r * 16;
  const int w_at = kXStage + share * kTiles * kW4TileBytes;
  const int s_at = kXStage + kGemmCodes + wave * 256;
  const uint32_t lds0 = lds_address(smem);
  // Steps past the end load the last one again, so that every step issues the same loads.
  auto load = [&](int step, int stage) {
    const int b = range.b0 + min(step, range.n - 1);
    const uint32_t to = lds0 + stage * kStage;
#pragma unroll
    for (int i = 0; i < kXLoads; ++i) async_load_1k(xs[i] + (int64_t)b * kBlock, to + (i * kGemmWaves + wave) * 1024);
#pragma unroll
    for (int i = 0; i < kWLoads; ++i)
      async_load_1k(ws[i] + (int64_t)b * kW4TileBytes, to + w_at + (half * kWLoads + i) * kW4TileBytes);
    async_load_256(ss + (b >> 2) * kW4ScaleTile + (b & 3) * 4, to + s_at);
  };
  auto store = [&](int c, v4f (&v)[kTiles]) {
    const int m = (first + c) * 16 + r;
    if (m >= mc) return;
#pragma unroll
    for (int t = 0; t < (GATEUP ? H : kTiles); ++t) {
      if (GATEUP) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[t][i] = silu_mul_fast(v[t][i], v[t + H][i]);
      }
      if (group(t) < groups) w4_store(p, p0 + m, group(t) * 16 + 4 * kq, v[t]);
    }
  };
  // A half without rows goes along with one part, of which it stores nothing.
  const int x_at = first * 16 * 2 * kBlock;
  constexpr int kMost = 2 * S / H;
  auto with = [&](auto parts_of) {
    constexpr int kCnt = decltype(parts_of)::value;
    w4_gemm_wave<kCnt, kTiles, kStages, kStage, kXLoads + kWLoads + 1>(smem, range.n, x_at, w_at, s_at, load, store);
  };
  if (kMost >= 5 && count == 5) with(std::integral_constant<int, kMost >= 5 ? 5 : 1>{});
  else if (kMost >= 4 && count == 4) with(std::integral_constant<int, kMost >= 4 ? 4 : 1>{});
  else if (kMost >= 3 && count == 3) with(std::integral_constant<int, kMost >= 3 ? 3 : 1>{});
  else if (kMost >= 2 && count == 2) with(std::integral_constant<int, kMost >= 2 ? 2 : 1>{});
  else with(std::integral_constant<int, 1>{});
}

template <int S, bool GATEUP>
moe_status_t launch_gemm(const W4Args& a, int64_t rows, hipStream_t stream) {
  constexpr int H = S <= 2 ? 1 : 2;
  const char* name = GATEUP ? "w4_gemm_gateup" : "w4_gemm";
  const int cols = GATEUP ? kGemmRows / 2 : kGemmRows;
  const int n_tiles = (a.N + cols - 1) / cols;
  const int64_t m_tiles = a.offsets ? rows / (32 * S) + (rows < a.E ? rows : (int64_t)a.E) : (rows + 32 * S - 1) / (32 * S);
  const bool dealt = m_tiles >= 4 * kXcd;
  const int64_t blocks = (dealt ? (m_tiles + kXcd - 1) / kXcd * kXcd : m_tiles) * n_tiles;
  if (blocks * std::max(1, a.splits) > w4_max_blocks(64 * kGemmWaves))
    return fail(MOE_ERR_UNSUPPORTED_SHAPE, "%s: too many rows and columns", name);
  MOE_LAUNCH(name, (w4_gemm_kernel<S, H, GATEUP>), dim3((unsigned)blocks, std::max(1, a.splits)), dim3(64 * kGemmWaves), 0,
             stream, a, rows, n_tiles, (int)dealt);
  return check_launch(name);
}

template <bool GATEUP>
moe_status_t gemm_by_rows(const W4Args& a, int64_t rows, hipStream_t stream) {
  // By the rows that an expert has on average: most experts in one tile, few of its parts empty.  (7168 x 2048, 256
  // experts, us a layer with S = 1 .. 5: 16 rows 1134 1162 1322 1377 1827, 48 rows 1860 1645 1702 1737 1998, 64 rows
  // 2210 2051 1893 1922 2153, 94 rows 2870 2779 2593 2369 2500, 128 rows 3700 3562 3508 3246 3008.)
  const int64_t mean = rows / a.E;
  if (mean <= 24) return launch_gemm<1, GATEUP>(a, rows, stream);
  if (mean <= 52) return launch_gemm<2, GATEUP>(a, rows, stream);
  if (mean <= 76) return launch_gemm<3, GATEUP>(a, rows, stream);
  if (mean <= 112) return launch_gemm<4, GATEUP>(a, rows, stream);
  return launch_gemm<5, GATEUP>(a, rows, stream);
}

}  // namespace

// How one matrix is cut: S of the tiles, and parts of K that a join adds up.  Taken by
// the time that each cut is expected to need, in us: rounds of 256 workgroups, each
// 4 and its steps (a step of 0.15 + 0.16 for every 16 rows, not less than 0.47:
// 20.6 us for 168 workgroups of 32 steps and 32 rows, 80 for 256 of 14 steps ... of 128
// rows), and for several parts a launch and their sums' way through memory.  Measured over 17 to 2048
// rows of 4096 x 6144, 7168 x 4096 and 2048 x 7168 it takes the fastest cut or one within 8 % of it.
W4Cut w4_gemm_cut(int64_t rows, int32_t K, int32_t N) {
  const int64_t n_tiles = ((int64_t)N + kGemmRows - 1) / kGemmRows;
  const int nb = K / kBlock;
  W4Cut best{4, 1};
  double best_us = 1e30;
  for (const int S : {1, 2, 4}) {
    const int64_t m_tiles = (rows + 32 * S - 1) / (32 * S);
    const double step = std::max(0.47, 0.15 + 0.01 * (double)even_tile_rows(rows, m_tiles));
    for (int parts = 1; parts <= w4_most_parts(rows) && parts * 3 <= std::max(nb, 3); ++parts) {
      const double rounds = (double)((m_tiles * n_tiles * parts + 255) / 256);
      const double us = rounds * (4.0 + (nb + parts - 1) / parts * step) +
                        (parts > 1 ? 4.0 + 8e-6 / 4.5 * (double)(parts * rows * N) : 0.0);
      if (us < best_us) {
        best_us = us;
        best = W4Cut{S, parts};
      }
    }
  }
  return best;
}

moe_status_t run_w4_gemm(const W4Args& a, bool gateup, int64_t rows, hipStream_t stream) {
  if (a.offsets) return gateup ? gemm_by_rows<true>(a, rows, stream) : gemm_by_rows<false>(a, rows, stream);
  switch (w4_gemm_cut(rows, a.K, a.N).tile) {
    case 1: return launch_gemm<1, false>(a, rows, stream);
    case 2: return launch_gemm<2, false>(a, rows, stream);
    default: return launch_gemm<4, false>(a, rows, stream);
  }
}

}  // namespace moe
