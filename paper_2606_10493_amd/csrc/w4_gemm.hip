// Products of many rows with 4-bit weights: an LDS-tiled bf16 GEMM that expands
// the weights in registers on their way from LDS to the matrix instruction.
//
// A workgroup takes a tile of up to 32 S activation rows against 128 TILES weight rows (1, 2 or 4)
// (GATEUP: 64 TILES of W_gate and the same rows of W_up).  Each of its eight waves, two to a
// SIMD, has 16 TILES weight rows and all activation rows, so that nothing is expanded
// twice and the expansion of one wave of a SIMD runs beside the products of the
// other.  How many 16-row parts the activation tile has is known when it is found, and
// each number has its own loop, so that an expert's rows are cut into equal tiles whose
// size follows them.
//
// Small tiles pay the expansion for few rows (an operand of 32 K takes four conversions of 6.5 cycles,
// 0.17 us of a step; with 32 activation rows a step takes 0.5 us), or are bound by the weights' stream where one row
// tile has them all (24 rows by 7168 x 65536 to fp32: 48 us, 5.3 TB/s); large ones by the matrix cores and the
// power that they draw (8192 rows by 7168 x 4096: 326 to 336 us, 1.43 to 1.48 PFLOP/s, where the library's product
// of bf16 weights takes 365; 4095 tokens of 8 of 256 experts of 7168 x 2048: gate and up 1.60 ms,
// 1.20 PFLOP/s, down 0.97 ms with 0.94 GB of sums).  With four waves, one to
// a SIMD, and tiles of 128 rows that layer took 4359 us, with eight and equal tiles 3077; up to six stages instead of three 50.4
// against 48.8 us (24 rows); the scales of four steps in one load as long as a step's.  The widest tiles
// (S = 5, TILES = 4) leave no register over: 28 bytes are kept in scratch memory, of which the loop of ten parts reads three
// or four values back a step.
//
// Steps of 128 K.  Activations (256 bytes a row), codes (1 KB a tile of 16 rows) and
// scales (one dword a row) go straight from global memory into LDS stages, one or
// two steps ahead, with one barrier a step; activation rows are gathered on the
// way.  The 16-byte piece c of an activation row lies at position c ^ row % 16, so
// that a quarter wave's reads fill all banks.  A step's barrier stands before the last
// products of the step in front of it, whose operands are in registers by then: the next
// codes are read and expanded beside them.
#include <algorithm>
#include <type_traits>

#include "w4.h"
#include "w4_rows.h"

namespace moe {

namespace {

constexpr int kGemmWaves = 8;
constexpr int kGemmScales = kGemmWaves * 256;  // of a stage: up to 64 rows' for each wave
constexpr int gemm_rows(int tiles) { return kGemmWaves * tiles * 16; }  // weight rows of a workgroup
constexpr int gemm_stage(int s, int tiles) { return 32 * s * 2 * kBlock + kGemmWaves * tiles * kW4TileBytes + kGemmScales; }
constexpr int gemm_stages(int s, int tiles) { return 3 * gemm_stage(s, tiles) <= 160 * 1024 ? 3 : 2; }

// async_load_1k of base + offset (base uniform, offset the lane's).
__device__ __forceinline__ void async_load_1k_at(const void* base, uint32_t offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(__builtin_amdgcn_readfirstlane((int)lds)), "v"(offset), "s"(base)
               : "memory");
}

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
__device__ __forceinline__ void w4_gemm_wave(const uint8_t* smem, int nb, int w_at, int s_at, Load load, Store store) {
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
        w4_bf16x8, *reinterpret_cast<const uint4*>(at + (c * 16 + r) * (2 * kBlock) + (((4 * j + kq) ^ r) * 16)));
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
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      constexpr int kLate = CNT * TILES <= 24 ? CNT : CNT <= 8 ? 3 : 2;  // parts whose last operands are read in front of the barrier
      const int now = j == 3 ? CNT - kLate : CNT;
#pragma unroll
      for (int c = 0; c < CNT; ++c) {
        if (c >= now) break;
        const w4_bf16x8 x = read_x(at, j, c);
#pragma unroll
        for (int t = 0; t < TILES; ++t) acc[t][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[j & 1][t], x, acc[t][c], 0, 0, 0);
      }
      if (j < 3) {
        expand(j + 1, w[(j + 1) & 1]);
        continue;
      }
      w4_bf16x8 late[kLate];
#pragma unroll
      for (int c = 0; c < kLate; ++c) late[c] = read_x(at, 3, now + c);
      // Step b + 1 has landed for every wave, and every wave has read all of step b, whose stage is loaded next.
      wait_async_and_barrier<(STAGES - 2) * LOADS>();
      read_codes(smem + next * STAGE_BYTES);
      load(b + STAGES, stage);
#pragma unroll
      for (int c = 0; c < kLate; ++c)
#pragma unroll
        for (int t = 0; t < TILES; ++t)
          acc[t][now + c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[1][t], late[c], acc[t][now + c], 0, 0, 0);
      expand(0, w[0]);
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
template <int S, int TILES, bool GATEUP>
__global__ __launch_bounds__(64 * kGemmWaves) void w4_gemm_kernel(W4Args p, int64_t rows, int n_tiles, int dealt) {
  constexpr int kXStage = 32 * S * 2 * kBlock;
  constexpr int kStage = gemm_stage(S, TILES), kStages = gemm_stages(S, TILES);
  constexpr int kRows = gemm_rows(TILES);
  constexpr int kXLoads = S;                      // a wave's a step: 8 S KB in all
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kStages * kStage];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
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
  // Tile t of the wave: 16-row group group(t) of its matrix (groups past the last are that one again).
  auto group = [&](int t) {
    if (GATEUP) return nt * (kRows / 32) + wave * (TILES / 2) + t % (TILES / 2);
    return nt * (kRows / 16) + wave * TILES + t;
  };
  auto up = [&](int t) { return GATEUP && t >= TILES / 2; };
  auto held = [&](int t) { return (int64_t)e * groups + min(group(t), groups - 1); };
  const uint8_t* ws[TILES];
#pragma unroll
  for (int t = 0; t < TILES; ++t) ws[t] = (up(t) ? p.w1 : p.w0) + held(t) * nb * kW4TileBytes;
  const int st = (lane >> 4) % TILES;  // lane 16 t + r: row r of tile t
  const uint8_t* ss = (up(st) ? p.s1 : p.s0) + held(st) * ((nb + 3) / 4) * kW4ScaleTile + r * 16;
  const int w_at = kXStage + wave * TILES * kW4TileBytes;
  const int s_at = kXStage + kGemmWaves * TILES * kW4TileBytes + wave * 256;
  const uint32_t lds0 = lds_address(smem);
  // Steps past the end load the last one again, so that every step issues the same loads.
  auto load = [&](int step, int stage) {
    const int b = range.b0 + min(step, range.n - 1);
    const uint32_t to = lds0 + stage * kStage;
#pragma unroll
    for (int i = 0; i < kXLoads; ++i) async_load_1k(xs[i] + (int64_t)b * kBlock, to + (i * kGemmWaves + wave) * 1024);
#pragma unroll
    for (int t = 0; t < TILES; ++t) async_load_1k_at(ws[t] + (int64_t)b * kW4TileBytes, lane * 16, to + w_at + t * kW4TileBytes);
    async_load_256(ss + (b >> 2) * kW4ScaleTile + (b & 3) * 4, to + s_at);
  };
  auto store = [&](int c, v4f (&v)[TILES]) {
    const int m = c * 16 + r;
    if (m >= mc) return;
#pragma unroll
    for (int t = 0; t < (GATEUP ? TILES / 2 : TILES); ++t) {
      if (GATEUP) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[t][i] = silu_mul_fast(v[t][i], v[t + TILES / 2][i]);
      }
      if (group(t) < groups) w4_store(p, p0 + m, group(t) * 16 + 4 * kq, v[t]);
    }
  };
  // The loop for this number of parts.
  auto with = [&](auto parts_of) {
    w4_gemm_wave<decltype(parts_of)::value, TILES, kStages, kStage, kXLoads + TILES + 1>(smem, range.n, w_at, s_at, load, store);
  };
  auto choose = [&](auto self, auto n) {
    constexpr int kN = decltype(n)::value;
    if constexpr (kN == 1) {
      with(n);
    } else {
      if (parts == kN) with(n);
      else self(self, std::integral_constant<int, kN - 1>{});
    }
  };
  choose(choose, std::integral_constant<int, 2 * S>{});
}

template <int S, int TILES, bool GATEUP>
moe_status_t launch_gemm(const W4Args& a, int64_t rows, hipStream_t stream) {
  const char* name = GATEUP ? "w4_gemm_gateup" : "w4_gemm";
  const int cols = gemm_rows(TILES) / (GATEUP ? 2 : 1);
  const int n_tiles = (int)(((int64_t)a.N + cols - 1) / cols);
  const int64_t m_tiles = a.offsets ? rows / (32 * S) + (rows < a.E ? rows : (int64_t)a.E) : (rows + 32 * S - 1) / (32 * S);
  const bool dealt = m_tiles >= 4 * kXcd;
  const int64_t blocks = (dealt ? (m_tiles + kXcd - 1) / kXcd * kXcd : m_tiles) * n_tiles;
  if (blocks * std::max(1, a.splits) > w4_max_blocks(64 * kGemmWaves))
    return fail(MOE_ERR_UNSUPPORTED_SHAPE, "%s: too many rows and columns", name);
  MOE_LAUNCH(name, (w4_gemm_kernel<S, TILES, GATEUP>), dim3((unsigned)blocks, std::max(1, a.splits)), dim3(64 * kGemmWaves), 0,
             stream, a, rows, n_tiles, (int)dealt);
  return check_launch(name);
}

template <bool GATEUP>
moe_status_t gemm_by_rows(const W4Args& a, int64_t rows, hipStream_t stream) {
  // S by the rows that an expert has on average: most experts in one tile, few of its parts empty.  Wide tiles read the
  // activations half as often, where the weights fill them and there are enough of them.  (7168 x 2048, 256 experts, us
  // a layer with S = 1 .. 5, TILES = 2: 32 rows 1473 1344 1362 1418 1846, 64 rows 2307 2087 1873 1902 2111, 128 rows 4203
  // 3582 3619 3305 3053; TILES = 4: 32 rows 1456 1226 1346 1347 1387, 64 rows 2302 1898 1706 1719 1719, 128 rows 4151
  // 3211 3251 2929 2786, 256 rows 7775 5996 5552 5366 5300.)
  const int64_t mean = rows / a.E;
  const int cols = gemm_rows(4) / (GATEUP ? 2 : 1);
  const int64_t n_tiles = ((int64_t)a.N + cols - 1) / cols;
  const bool wide = n_tiles * cols * 7 <= (int64_t)a.N * 8 && std::min<int64_t>(rows, a.E) * n_tiles >= 256;
  if (wide && mean > 12) {
    if (mean <= 52) return launch_gemm<2, 4, GATEUP>(a, rows, stream);
    if (mean <= 72) return launch_gemm<3, 4, GATEUP>(a, rows, stream);
    if (mean <= 104) return launch_gemm<4, 4, GATEUP>(a, rows, stream);
    return launch_gemm<5, 4, GATEUP>(a, rows, stream);
  }
  if (mean <= 24) return launch_gemm<1, 2, GATEUP>(a, rows, stream);
  if (mean <= 52) return launch_gemm<2, 2, GATEUP>(a, rows, stream);
  if (mean <= 76) return launch_gemm<3, 2, GATEUP>(a, rows, stream);
  if (mean <= 112) return launch_gemm<4, 2, GATEUP>(a, rows, stream);
  return launch_gemm<5, 2, GATEUP>(a, rows, stream);
}

}  // namespace

// How one matrix is cut, by the time that each cut is expected to need, in us: rounds of
// 256 workgroups, each 4 and its steps, a step 0.15 and 0.0115 an activation row with
// narrow tiles, 0.3 and 0.019 with wide ones, 0.31 with the smallest; and for several parts of K a launch and
// their sums' way through memory.  (20.3 us for 168 workgroups of 32 steps of 29 rows, 53.5 for 192 of 32 of 128; wide, 92.5 for
// 192 of 32 of 128 rows and 338 for 512 of 56.  The smallest, 128 weight rows by 32, beside 256 by 32 in parts of K: 6.0
// against 7.8 us for 100 rows by 1024 x 1536, 9.1 against 11.7 for 2048 x 7168, 14.0 against 16.7 for 4096 x
// 6144; 128 by 64 instead: 35.5 against 33.0 for 512 rows by 7168 x 4096.)
W4Cut w4_gemm_cut(int64_t rows, int32_t K, int32_t N) {
  const int nb = K / kBlock;
  constexpr struct {
    int S, tiles;
    double step, row;
  } kKinds[] = {{1, 1, 0.31, 0.0},   {1, 2, 0.15, 0.0115}, {2, 2, 0.15, 0.0115}, {4, 2, 0.15, 0.0115},
                {3, 4, 0.3, 0.019}, {4, 4, 0.3, 0.019},   {5, 4, 0.3, 0.019}};
  W4Cut best{4, 2, 1};
  double best_us = 1e30;
  for (const auto& k : kKinds) {
    const int64_t m_tiles = (rows + 32 * k.S - 1) / (32 * k.S), n_tiles = ((int64_t)N + gemm_rows(k.tiles) - 1) / gemm_rows(k.tiles);
    const double step = k.step + k.row * (double)even_tile_rows(rows, m_tiles);
    for (int parts = 1; parts <= w4_most_parts(rows) && parts * 3 <= std::max(nb, 3); ++parts) {
      const double rounds = (double)((m_tiles * n_tiles * parts + 255) / 256);
      const double us = rounds * (4.0 + (nb + parts - 1) / parts * step) +
                        (parts > 1 ? 4.0 + 8e-6 / 4.5 * (double)(parts * rows * N) : 0.0);
      if (us < best_us) {
        best_us = us;
        best = W4Cut{k.S, k.tiles, parts};
      }
    }
  }
  return best;
}

moe_status_t run_w4_gemm(const W4Args& a, bool gateup, int64_t rows, hipStream_t stream) {
  if (a.offsets) return gateup ? gemm_by_rows<true>(a, rows, stream) : gemm_by_rows<false>(a, rows, stream);
  const W4Cut cut = w4_gemm_cut(rows, a.K, a.N);
  switch (10 * cut.tiles + cut.S) {
    case 11: return launch_gemm<1, 1, false>(a, rows, stream);
    case 21: return launch_gemm<1, 2, false>(a, rows, stream);
    case 22: return launch_gemm<2, 2, false>(a, rows, stream);
    case 24: return launch_gemm<4, 2, false>(a, rows, stream);
    case 43: return launch_gemm<3, 4, false>(a, rows, stream);
    case 44: return launch_gemm<4, 4, false>(a, rows, stream);
    default: return launch_gemm<5, 4, false>(a, rows, stream);
  }
}

}  // namespace moe
