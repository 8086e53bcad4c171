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

constexpr int kFewMaxRows = 2048;  // rows of all experts whose tiles w4_few lists in LDS

constexpr int kSortSlots = 64;  // slots that a wave sorts by itself

// The sort of moe_permute for up to 64 slots, one a lane, by one wave: src[p] = slot at
// sorted position p, `place` the lane's position, and the row tiles of 16 as
// list_row_tiles lists them (returned: how many).  Slots whose id lies outside [0, E)
// come last and belong to no tile.  Every lane compares with every slot.
__device__ __forceinline__ int sort_slots(const int32_t* __restrict__ ids, int slots, int E, int2* list, int* src, int& place) {
  const int lane = threadIdx.x & 63;
  const int id = lane < slots ? ids[lane] : -1;
  const bool ok = id >= 0 && id < E;
  const int key = ok ? id : INT32_MAX;
  int less = 0, before = 0, same = 0;
  for (int i0 = 0; i0 < slots; i0 += 8) {  // (lanes behind the last slot count as bad ids behind it)
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int other = __builtin_amdgcn_readlane(key, i0 + u);
      less += other < key ? 1 : 0;
      same += other == key ? 1 : 0;
      before += other == key && i0 + u < lane ? 1 : 0;
    }
  }
  place = less + before;
  const bool begins = ok && before % 16 == 0;
  const unsigned long long all = __ballot(begins);
  int rank = 0;
  const int begin_at = begins ? place : INT32_MAX;
  for (int i0 = 0; i0 < slots; i0 += 8) {
#pragma unroll
    for (int u = 0; u < 8; ++u) rank += __builtin_amdgcn_readlane(begin_at, i0 + u) < place ? 1 : 0;
  }
  if (lane < slots) src[place] = lane;
  if (begins) list[rank] = make_int2(place, id | min(16, same - before) << 16);
  return __popcll(all);
}

// MOE_DEV_* bits of the slots' ids, known to every lane.
__device__ __forceinline__ int slot_errors(const int32_t* __restrict__ ids, int slots, int topk, int E) {
  const int lane = threadIdx.x & 63;
  const int id = lane < slots ? ids[lane] : -1;
  const int token = lane / topk * topk;  // the token's first slot
  bool twice = false;
  for (int i0 = 0; i0 < slots; i0 += 8) {
#pragma unroll
    for (int u = 0; u < 8; ++u)
      twice |= i0 + u >= token && i0 + u < lane && lane < slots && __builtin_amdgcn_readlane(id, i0 + u) == id;
  }
  const bool bad = lane < slots && (id < 0 || id >= E);
  return (__any(bad) ? MOE_DEV_BAD_EXPERT_ID : 0) | (__any(twice && !bad) ? MOE_DEV_DUP_EXPERT_ID : 0);
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
