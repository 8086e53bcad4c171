// The down projection and the combine of a few slots with 4-bit weights in one
// launch: a workgroup computes 16 output columns for every slot and combines them
// per token in LDS, so that the fp32 expert rows are not written.
//
// Wave w takes the row tiles w, w + 8, ... (a few slots have about as many active
// experts) and streams their 16 weight rows over all of K with two halves of kDownBlocks K
// blocks in flight; the slots' rows of h lie in LDS.  One token of 8 experts of 7168 x 2048:
// 62 MB in 14 us, 7 of them for the launch and the dependent loads (the list, the weights) before the
// stream and the combine behind it; with a combine of its own the layer took 7 us more.  The sums of a row tile are
// the same as w4_few's but for their order in K; the combine is the definition's order
// (see moe_combine).  Three values are kept in scratch memory, outside of the product loops.
#include "w4.h"
#include "w4_rows.h"

namespace moe {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kDownWaves = 8;
constexpr int kDownBlocks = 4;            // K blocks that are loaded together
constexpr int kDownFirst = 2 * (kDownBlocks + kDownBlocks / 4);  // loads of a wave's first weights
constexpr int kDownBytes = 80 * 1024;     // of LDS

struct W4DownArgs {
  const uint16_t* h;    // bf16 [slots, K], sorted
  const int2* list;     // row tiles, their number in entry kSortSlots
  const uint8_t *w, *s;  // packed [E, N, K]
  int slots, tokens, topk, N, K;
  const int32_t* dest_row;
  const float* topk_w;
  uint16_t* out;        // bf16 [tokens, N]
};

// LDS: the rows of h (whole loads of 1 KB; the 16-byte piece c of row i lies at c ^ i % 16, so that rows begin on other
// banks), then y.
constexpr int64_t down_h_bytes(int K, int slots) { return ((int64_t)slots * K * 2 + 1023) / 1024 * 1024; }
constexpr int64_t down_bytes(int K, int slots) { return down_h_bytes(K, slots) + slots * 64; }

__global__ __launch_bounds__(64 * kDownWaves, 4) void w4_down_combine_kernel(W4DownArgs p) {
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  float* y = reinterpret_cast<float*>(lds + down_h_bytes(p.K, p.slots));  // [slots][16]
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, kq = lane >> 4;
  const int nb = p.K / kBlock, groups = p.N / 16, chunks = (nb + 3) / 4;
  // (Loaded in front of the asm below, the list comes as scalars and waits for no other load.)
  const int2 count = p.list[kSortSlots], own = p.list[wave];
  // The rows of h go out first, so that they are there when the first weights are.
  const int pieces = p.K / 8;
  {
    const int all = p.slots * pieces;
    const uint32_t to = lds_address(lds);
    for (int i = wave * 64; i < all; i += kDownWaves * 64) {
      const int at = min(i + lane, all - 1), row = at / pieces;
      async_load_1k(p.h + (int64_t)row * p.K + ((at - row * pieces) ^ (row & 15)) * 8, to + i * 16);
    }
  }
  const int n = __builtin_amdgcn_readfirstlane(count.x);

  struct Blocks {
    u32x4 w[kDownBlocks];
    u32x4 s[kDownBlocks / 4];
  };
  int e = 0, p0 = 0, m = 0;
  const uint8_t *wt = p.w, *st = p.s;
  auto point = [&](int2 tile) {
    const int em = __builtin_amdgcn_readfirstlane(tile.y);
    p0 = __builtin_amdgcn_readfirstlane(tile.x);
    e = em & 0xffff;
    m = em >> 16;
    const int64_t g = (int64_t)e * groups + blockIdx.x;
    wt = p.w + g * nb * kW4TileBytes + lane * 16;
    st = p.s + g * chunks * kW4ScaleTile + r * 16;
  };
  auto load = [&](int b, Blocks& q) {  // blocks past the last are that one again
#pragma unroll
    for (int u = 0; u < kDownBlocks / 4; ++u)
      q.s[u] = *reinterpret_cast<const u32x4*>(st + min((b >> 2) + u, chunks - 1) * kW4ScaleTile);
#pragma unroll
    for (int u = 0; u < kDownBlocks; ++u)
      q.w[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(wt + (int64_t)min(b + u, nb - 1) * kW4TileBytes));
  };
  Blocks q0, q1;
  if (wave < n) {
    point(own);
    load(0, q0);
    load(kDownBlocks, q1);
  }
  // A wave's loads of h are its oldest.
  if (wave < n) wait_async_and_barrier<kDownFirst>();
  else wait_async_and_barrier<0>();

  for (int a = wave; a < n; a += kDownWaves) {
    if (a != wave) {
      point(p.list[a]);
      load(0, q0);
      load(kDownBlocks, q1);
    }
    const int row = p0 + min(r, m - 1);
    const uint8_t* x = lds + row * (2 * p.K);
    const int turn = row & 15;
    v4f acc[2] = {v4f{0.f, 0.f, 0.f, 0.f}, v4f{0.f, 0.f, 0.f, 0.f}};  // of even and odd blocks
    auto block = [&](int b, int u, const Blocks& q) {
      w4_bf16x8 xu[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        xu[j] = __builtin_bit_cast(w4_bf16x8, *reinterpret_cast<const uint4*>(x + ((4 * j + kq) ^ turn) * 16 + (b + u) * (2 * kBlock)));
#pragma unroll
      for (int j = 0; j < 4; ++j)
        acc[u & 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w4_expand(q.w[u][j], w4_scale(q.s[u / 4][u % 4], j)), xu[j], acc[u & 1],
                                                             0, 0, 0);
    };
    auto multiply = [&](int b, const Blocks& q) {
      if (b + kDownBlocks <= nb) {  // (one basic block, whose reads of h run ahead of the products)
#pragma unroll
        for (int u = 0; u < kDownBlocks; ++u) block(b, u, q);
      } else {
#pragma unroll
        for (int u = 0; u < kDownBlocks; ++u)
          if (b + u < nb) block(b, u, q);
      }
    };
    for (int b = 0; b < nb; b += 2 * kDownBlocks) {
      multiply(b, q0);
      if (b + 2 * kDownBlocks < nb) load(b + 2 * kDownBlocks, q0);
      if (b + kDownBlocks >= nb) break;
      multiply(b + kDownBlocks, q1);
      if (b + 3 * kDownBlocks < nb) load(b + 3 * kDownBlocks, q1);
    }
    if (r < m) *reinterpret_cast<v4f*>(y + (p0 + r) * 16 + 4 * kq) = acc[0] + acc[1];
  }
  __syncthreads();
  // Tokens' sums in slot order, products and sums rounded separately.
  for (int i = threadIdx.x; i < p.tokens * 16; i += 64 * kDownWaves) {
#pragma clang fp contract(off)
    const int t = i / 16, c = i % 16;
    float sum = 0.0f;
    for (int j = 0; j < p.topk; ++j) sum = sum + p.topk_w[t * p.topk + j] * y[p.dest_row[t * p.topk + j] * 16 + c];
    p.out[(int64_t)t * p.N + blockIdx.x * 16 + c] = f32_to_bf16_rne(sum);
  }
}

}  // namespace

bool w4_down_combine_fits(int32_t K, int slots) {
  return slots <= kSortSlots && down_bytes(K, slots) <= kDownBytes;
}

moe_status_t run_w4_down_combine(const moe_dims_t& d, int tokens, const uint16_t* h, const W4Slots& s, const uint8_t* w,
                                 const uint8_t* w_s, const float* topk_w, uint16_t* out, hipStream_t stream) {
  const int slots = tokens * d.topk;
  const W4DownArgs a{h, s.list, w, w_s, slots, tokens, d.topk, d.hidden, d.inter, s.dest_row, topk_w, out};
  MOE_LAUNCH("w4_down_combine", w4_down_combine_kernel, dim3((unsigned)(d.hidden / 16)), dim3(64 * kDownWaves),
             (size_t)down_bytes(d.inter, slots), stream, a);
  return check_launch("w4_down_combine");
}

}  // namespace moe
