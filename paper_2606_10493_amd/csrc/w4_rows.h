// Finding the expert and its rows that a workgroup works for, by one wave (every
// wave does it for itself: no barrier).  Offsets are cut to 0 .. rows.
#pragma once

#include "common.h"

namespace moe {

struct ExpertRows {
  int e, p0, m;  // expert (-1: there is none), first row, rows
};

// The row tiles of 256 experts, c0 + 64 c + lane being the lane's in part c: their
// first rows, rows, and in `upto` the tiles of all 256 up to and with it.  The
// offsets go out together, so that this costs one round trip.
struct TileCounts {
  int lo[4], n[4], upto[4], all;
};

__device__ __forceinline__ TileCounts count_tiles(const int32_t* __restrict__ offsets, int E, int c0, int tile, int rows) {
  const int lane = threadIdx.x & 63;
  TileCounts t;
  int hi[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const int x = c0 + 64 * c + lane;
    t.lo[c] = offsets[min(x, E)];
    hi[c] = offsets[min(x + 1, E)];
  }
  t.all = 0;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    t.lo[c] = min(max(t.lo[c], 0), rows);
    t.n[c] = c0 + 64 * c + lane < E ? max(min(hi[c], rows) - t.lo[c], 0) : 0;
    int x = (int)(((int64_t)t.n[c] + tile - 1) / tile);
    // Inclusive sum over the lanes: neighbours, rows of 16 and halves by register moves.
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);   // row_shr:1
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);   // row_shr:2
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);   // row_shr:4
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);   // row_shr:8
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast:15 into rows 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast:31 into rows 2 and 3
    t.upto[c] = t.all + x;
    t.all += __builtin_amdgcn_readlane(x, 63);
  }
  return t;
}

// The row tiles of all experts in order, `tile` rows each but for an expert's last, as
// {first row, expert | rows << 16}, those before `most`; returns how many there are.
// tile <= 256, E <= 65536.  For the lanes of one wave.
__device__ __forceinline__ int list_row_tiles(const int32_t* __restrict__ offsets, int E, int tile, int rows, int most, int2* list) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int c0 = 0; c0 < E; c0 += 256) {
    const TileCounts t = count_tiles(offsets, E, c0, tile, rows);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int own = (t.n[c] + tile - 1) / tile;
      for (int i = 0; i < own; ++i) {
        const int at = before + t.upto[c] - own + i;
        if (at < most) list[at] = make_int2(t.lo[c] + i * tile, (c0 + 64 * c + lane) | min(tile, t.n[c] - i * tile) << 16);
      }
    }
    before += t.all;
  }
  return min(before, most);
}

// Rows of each of `tiles` tiles that share n rows evenly, in parts of 16 (the last
// tile may hold fewer, or none).
__host__ __device__ __forceinline__ int64_t even_tile_rows(int64_t n, int64_t tiles) {
  return ((n + tiles - 1) / tiles + 15) / 16 * 16;
}

// The a-th of the tiles that share their expert's rows evenly, the fewest of at most
// `tile` rows (a multiple of 16).
__device__ __forceinline__ ExpertRows find_even_tile(const int32_t* __restrict__ offsets, int E, int a, int tile, int rows) {
  for (int c0 = 0; c0 < E; c0 += 256) {
    const TileCounts t = count_tiles(offsets, E, c0, tile, rows);
    if (a < t.all) {
      ExpertRows found{-1, 0, 0};
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const unsigned long long holds = __ballot(a < t.upto[c]);
        if (found.e < 0 && holds) {
          const int at = __ffsll((long long)holds) - 1;
          const int n = __builtin_amdgcn_readlane(t.n[c], at);
          const int tiles = (n + tile - 1) / tile;
          const int part = (int)even_tile_rows(n, tiles);
          const int skip = (tiles - (__builtin_amdgcn_readlane(t.upto[c], at) - a)) * part;
          found = ExpertRows{skip < n ? c0 + 64 * c + at : -2, __builtin_amdgcn_readlane(t.lo[c], at) + skip, min(part, n - skip)};
          if (found.e == -2) return ExpertRows{-1, 0, 0};
        }
      }
      return found;
    }
    a -= t.all;
  }
  return ExpertRows{-1, 0, 0};
}

}  // namespace moe
