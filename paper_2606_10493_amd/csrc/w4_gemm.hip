// Products of many rows with 4-bit weights: an LDS-tiled bf16 GEMM that expands
// the weights in registers on their way from LDS to the matrix instruction.
//
// A workgroup of four waves takes 16 MT activation rows against 256 weight rows
// (GATEUP: 128 of W_gate and the same 128 of W_up), a wave 64 of them (32 and
// 32) against all activation rows: no weight is expanded twice in a workgroup.
// Steps of 128 K.  Activations (256 bytes a row), codes (a wave's four 1 KB
// tiles) and scales (one dword a row) go straight from global memory into three
// LDS stages, two steps ahead, with one barrier a step; activation rows are
// gathered on the way.  The 16-byte piece c of an activation row lies at position
// c ^ row % 16, so that a quarter wave's reads fill all banks.
#include "w4.h"
#include "w4_rows.h"

namespace moe {

namespace {

constexpr int kGemmWaves = 4;
constexpr int kGemmTiles = 4;  // 16-row weight tiles of a wave
constexpr int kGemmStages = 3;
constexpr int kGemmRows = kGemmWaves * kGemmTiles * 16;  // weight rows of a workgroup
constexpr int kGemmWaveStage = kGemmTiles * kW4TileBytes + kGemmTiles * 64;  // codes, then scales

// async_load_1k's counterpart for 4 bytes a lane.
__device__ __forceinline__ void async_load_256(const void* src, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
               :
               : "s"(__builtin_amdgcn_readfirstlane((int)lds)), "v"(src)
               : "memory");
}

template <int MT, bool GATEUP>
__global__ __launch_bounds__(64 * kGemmWaves) void w4_gemm_kernel(W4Args p, int64_t rows, int n_tiles) {
  constexpr int kXStage = 16 * MT * 2 * kBlock;
  constexpr int kStage = kXStage + kGemmWaves * kGemmWaveStage;
  constexpr int kLoads = MT + kGemmTiles + 1;  // a wave's a step
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kGemmStages * kStage];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, kq = lane >> 4;
  const int nb = p.K / kBlock, groups = p.N / 16;
  const int64_t a = blockIdx.x / n_tiles;
  const int nt = (int)(blockIdx.x % n_tiles);

  int e = 0, mc;
  int64_t p0;
  if (p.offsets) {
    const ExpertRows ref = find_row_tile(p.offsets, p.E, (int)a, 16 * MT, (int)rows);
    if (ref.e < 0) return;  // the whole workgroup
    e = ref.e;
    p0 = ref.p0;
    mc = ref.m;
  } else {
    p0 = a * 16 * MT;
    mc = (int)min((int64_t)16 * MT, rows - p0);
  }

  // Sources.  Load i of the activations takes rows 16 i + 4 wave + lane / 16.
  const uint16_t* xs[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int m = 16 * i + 4 * wave + (lane >> 4);
    int64_t row = p0 + min(m, mc - 1);  // rows past the tile's end read a valid one, and are not stored
    if (p.sorted_src) {
      row = p.sorted_src[row] / p.topk;
      if (row < 0 || row >= p.x_rows) row = 0;
    }
    xs[i] = p.x + row * p.x_stride + (((lane & 15) ^ (m & 15)) * 8);
  }
  // Tile t of the wave: 16-row group `group(t)` of its matrix (groups past the last are that one again).
  auto group = [&](int t) {
    if (GATEUP) return nt * (kGemmRows / 32) + wave * 2 + (t & 1);
    return nt * (kGemmRows / 16) + wave * kGemmTiles + t;
  };
  const uint8_t* ws[kGemmTiles];
#pragma unroll
  for (int t = 0; t < kGemmTiles; ++t)
    ws[t] = (GATEUP && t >= 2 ? p.w1 : p.w0) + ((int64_t)e * groups + min(group(t), groups - 1)) * nb * kW4TileBytes + lane * 16;
  const uint8_t* ss;  // lane 16 t + r: row r of tile t
  {
    const int t = lane >> 4;
    ss = (GATEUP && t >= 2 ? p.s1 : p.s0) + ((int64_t)e * groups + min(group(t), groups - 1)) * ((nb + 3) / 4) * kW4ScaleTile + r * 16;
  }
  const uint32_t lds0 = lds_address(smem);
  // Steps past the end load the last one again, so that every step issues the same loads.
  auto load = [&](int step, int stage) {
    const int b = min(step, nb - 1);
    const uint32_t to = lds0 + stage * kStage;
#pragma unroll
    for (int i = 0; i < MT; ++i) async_load_1k(xs[i] + (int64_t)b * kBlock, to + (i * kGemmWaves + wave) * 1024);
    const uint32_t own = to + kXStage + wave * kGemmWaveStage;
#pragma unroll
    for (int t = 0; t < kGemmTiles; ++t) async_load_1k(ws[t] + (int64_t)b * kW4TileBytes, own + t * kW4TileBytes);
    async_load_256(ss + (b >> 2) * kW4ScaleTile + (b & 3) * 4, own + kGemmTiles * kW4TileBytes);
  };

  v4f acc[kGemmTiles][MT];
#pragma unroll
  for (int t = 0; t < kGemmTiles; ++t)
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) acc[t][mt] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < kGemmStages - 1; ++s) load(s, s);
  int stage = 0, fill = kGemmStages - 1;
  for (int b = 0; b < nb; ++b) {
    // Step b has landed for every wave, and every wave has read step b - 1, whose stage is loaded next.
    wait_async_and_barrier<(kGemmStages - 2) * kLoads>();
    load(b + kGemmStages - 1, fill);
    const uint8_t* at = smem + stage * kStage;
    const uint8_t* own = at + kXStage + wave * kGemmWaveStage;
    uint4 raw[kGemmTiles];
    uint32_t sc[kGemmTiles];
#pragma unroll
    for (int t = 0; t < kGemmTiles; ++t) {
      raw[t] = *reinterpret_cast<const uint4*>(own + t * kW4TileBytes + lane * 16);
      sc[t] = *reinterpret_cast<const uint32_t*>(own + kGemmTiles * kW4TileBytes + 64 * t + 4 * r);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      w4_bf16x8 w[kGemmTiles];
#pragma unroll
      for (int t = 0; t < kGemmTiles; ++t) {
        const uint32_t codes = j == 0 ? raw[t].x : j == 1 ? raw[t].y : j == 2 ? raw[t].z : raw[t].w;
        w[t] = w4_expand(codes, w4_scale(sc[t], j));
      }
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        const w4_bf16x8 x = __builtin_bit_cast(
            w4_bf16x8, *reinterpret_cast<const uint4*>(at + (mt * 16 + r) * (2 * kBlock) + (((4 * j + kq) ^ r) * 16)));
#pragma unroll
        for (int t = 0; t < kGemmTiles; ++t) acc[t][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[t], x, acc[t][mt], 0, 0, 0);
      }
    }
    stage = stage + 1 == kGemmStages ? 0 : stage + 1;
    fill = fill + 1 == kGemmStages ? 0 : fill + 1;
  }
  // No load may reach LDS after the workgroup has ended.
  wait_async_and_barrier<0>();

  // Lane 16 kq + r holds outputs 4 kq .. 4 kq + 3 of each tile for row r of each 16.
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int m = mt * 16 + r;
    if (m >= mc) continue;
#pragma unroll
    for (int t = 0; t < (GATEUP ? 2 : kGemmTiles); ++t) {
      v4f v = acc[t][mt];
      if (GATEUP) {
#pragma unroll
        for (int c = 0; c < 4; ++c) v[c] = silu_mul_fast(v[c], acc[t + 2][mt][c]);
      }
      if (group(t) < groups) w4_store(p, p0 + m, group(t) * 16 + 4 * kq, v);
    }
  }
}

template <int MT, bool GATEUP>
moe_status_t launch_gemm(const W4Args& a, int64_t rows, hipStream_t stream) {
  const char* name = GATEUP ? "w4_gemm_gateup" : "w4_gemm";
  const int cols = GATEUP ? kGemmRows / 2 : kGemmRows;
  const int n_tiles = (a.N + cols - 1) / cols;
  const int64_t m_tiles = a.offsets ? rows / (16 * MT) + (rows < a.E ? rows : (int64_t)a.E) : (rows + 16 * MT - 1) / (16 * MT);
  if (m_tiles * n_tiles > w4_max_blocks(64 * kGemmWaves))
    return fail(MOE_ERR_UNSUPPORTED_SHAPE, "%s: too many rows and columns", name);
  MOE_LAUNCH(name, (w4_gemm_kernel<MT, GATEUP>), dim3((unsigned)(m_tiles * n_tiles)), dim3(64 * kGemmWaves), 0, stream, a, rows,
             n_tiles);
  return check_launch(name);
}

template <bool GATEUP>
moe_status_t gemm_by_rows(const W4Args& a, int64_t rows, hipStream_t stream) {
  const int64_t mean = a.offsets ? rows / a.E : rows;  // rows a matrix
  if (mean <= 32) return launch_gemm<2, GATEUP>(a, rows, stream);
  if (mean <= 96) return launch_gemm<4, GATEUP>(a, rows, stream);
  return launch_gemm<8, GATEUP>(a, rows, stream);
}

}  // namespace

moe_status_t run_w4_gemm(const W4Args& a, bool gateup, int64_t rows, hipStream_t stream) {
  return gateup ? gemm_by_rows<true>(a, rows, stream) : gemm_by_rows<false>(a, rows, stream);
}

}  // namespace moe
