// Finding the expert and its rows that a workgroup works for, by one wave (every
// wave does it for itself: no barrier).  Offsets are cut to 0 .. rows.
#pragma once

#include "common.h"

namespace moe {

struct ExpertRows {
  int e, p0, m;  // expert (-1: there is none), first row, rows
};

// Lane l's expert c0 + l: its first row and the row behind its last.
__device__ __forceinline__ void expert_span(const int32_t* __restrict__ offsets, int E, int x, int rows, int& lo, int& hi) {
  lo = min(max(offsets[min(x, E)], 0), rows);
  hi = x < E ? min(max(offsets[min(x + 1, E)], lo), rows) : lo;
}

// The a-th of the experts that have m_lo to m_hi rows.  The offsets of 256 experts
// go out together, so that the search costs one round trip.
__device__ __forceinline__ ExpertRows find_expert(const int32_t* __restrict__ offsets, int E, int a, int m_lo, int m_hi, int rows) {
  const int lane = threadIdx.x & 63;
  ExpertRows found{-1, 0, 0};
  for (int c0 = 0; c0 < E && found.e < 0; c0 += 256) {
    int lo[4], hi[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) expert_span(offsets, E, c0 + 64 * c + lane, rows, lo[c], hi[c]);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int n = hi[c] - lo[c];
      unsigned long long on = __ballot(n >= m_lo && n <= m_hi && n > 0);
      const int count = __popcll(on);
      if (found.e < 0 && a < count) {
        for (int i = 0; i < a; ++i) on &= on - 1ull;
        const int at = __ffsll((long long)on) - 1;
        found = ExpertRows{c0 + 64 * c + at, __shfl(lo[c], at), __shfl(n, at)};
      }
      a -= count;
    }
  }
  return found;
}

// The a-th tile of `tile` rows over all experts in order (an expert's last tile may
// hold fewer rows).
__device__ __forceinline__ ExpertRows find_row_tile(const int32_t* __restrict__ offsets, int E, int64_t a, int tile, int rows) {
  const int lane = threadIdx.x & 63;
  ExpertRows found{-1, 0, 0};
  for (int c0 = 0; c0 < E && found.e < 0; c0 += 256) {
    int lo[4], hi[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) expert_span(offsets, E, c0 + 64 * c + lane, rows, lo[c], hi[c]);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int own = (int)(((int64_t)hi[c] - lo[c] + tile - 1) / tile);
      int n = own;  // becomes the tiles of the experts up to this lane's
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(n, d);
        if (lane >= d) n += y;
      }
      const unsigned long long holds = __ballot(a < n);
      if (found.e < 0 && holds) {
        const int at = __ffsll((long long)holds) - 1;
        const int first = __shfl(lo[c], at) + ((int)a - __shfl(n - own, at)) * tile;
        found = ExpertRows{c0 + 64 * c + at, first, min(tile, __shfl(hi[c], at) - first)};
      }
      a -= __shfl(n, 63);
    }
  }
  return found;
}

}  // namespace moe
