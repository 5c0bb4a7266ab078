// attend.hpp -- what the attention kernels over a paged cache share: their arguments, the
// drafts a token sees, and the joining of a sequence's parts.
#pragma once

#include <algorithm>

#include "cache.hpp"

namespace moe {
namespace cache {
namespace {

constexpr int kMaxSplit = 64;    // the joining wave holds one part's statistics per lane

struct AttendArgs {
  Batch b;
  const void *q, *kc, *vc;
  void* out;
  float *part, *stat;   // [n_split][rows][D] sums and [n_split][rows][2] (maximum, sum) of the parts
  const uint64_t* mask;
  int64_t ld_q, ld_out;
  float scale2;         // |scale| * log2(e): scores are powers of two
  uint32_t flip;        // 0x80008000 for a negative scale, which turns the queries' signs
  int n_q_heads, group, mask_words, n_split, part_tiles, row_blocks, units;
};

// Tiles of one part of a sequence's keys: equal parts, as many as it takes for none to be
// longer than the longest sequence's (as the host knows it), n_split at most.
__device__ __forceinline__ int tiles_per_part(const AttendArgs& a, int tiles) {
  const int parts = min(a.n_split, (tiles + a.part_tiles - 1) / a.part_tiles);
  return (tiles + parts - 1) / max(parts, 1);
}

// Bits of the 8 drafts from d0 on (d0 may be negative: slots of cached tokens, seen by
// all) that token i (row t) sees, of its sequence's n.
__device__ __forceinline__ uint32_t seen8(const AttendArgs& a, int64_t t, int i, int n, int d0) {
  if (d0 <= -8) return 0xFFu;
  const int d = max(d0, 0), left = n - d;
  uint32_t bits = 0;
  if (left > 0) {
    if (a.mask) {
      const uint64_t* m = a.mask + t * a.mask_words;
      const int w = d >> 6, sh = d & 63;
      if (w < a.mask_words) bits = static_cast<uint32_t>(m[w] >> sh);
      if (sh > 56 && w + 1 < a.mask_words) bits |= static_cast<uint32_t>(m[w + 1] << (64 - sh));
    } else if (i >= d) {
      bits = i - d >= 7 ? 0xFFu : (2u << (i - d)) - 1;
    }
    if (left < 8) bits &= (1u << left) - 1;
  }
  if (d0 < 0) bits = bits << -d0 | ((1u << -d0) - 1);
  return bits & 0xFFu;
}

// Joins the parts of each (new token, query head): WPR waves take every WPR-th part, lanes
// side by side over the channels, and are added in wave order.
template <int TYPE, int D, int TILE, int WPR>
__global__ void __launch_bounds__(256) join_kernel(AttendArgs a) {
  typedef elem_t<TYPE> E;
  constexpr int C = D / kWave, U = 4;   // U parts' loads at once
  __shared__ float sums[4][D];
  const int64_t all_rows = static_cast<int64_t>(a.b.n_seqs) * a.b.max_new * a.n_q_heads;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t row = WPR == 4 ? blockIdx.x : static_cast<int64_t>(blockIdx.x) * 4 + wave;
  if (row >= all_rows) return;
  const int head = static_cast<int>(row % a.n_q_heads);
  const int64_t tok = row / a.n_q_heads;
  const int s = static_cast<int>(tok / a.b.max_new), i = static_cast<int>(tok % a.b.max_new);
  bool ok;
  const Seq q = sequence(a.b, s, ok);
  if (i >= q.n) return;
  const int tiles = (q.len + q.n + TILE - 1) / TILE, per = tiles_per_part(a, tiles);
  const int parts = (tiles + per - 1) / per;
  float m = -INFINITY, l = 0.f;
  if (lane < parts) {
    m = a.stat[2 * (lane * all_rows + row)];
    l = a.stat[2 * (lane * all_rows + row) + 1];
  }
  float x[C];
#pragma unroll
  for (int c = 0; c < C; c++) x[c] = 0.f;
  float top = m;
  for (int w = 32; w; w >>= 1) top = fmaxf(top, __shfl_xor(top, w));
  const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - top) * a.scale2);
  const float sum = wave_sum(l * f);
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
  for (int p0 = WPR == 4 ? wave : 0; p0 < parts; p0 += WPR * U) {
    float y[U][C];
#pragma unroll
    for (int u = 0; u < U; u++)
#pragma unroll
      for (int c = 0; c < C; c++) y[u][c] = p0 + WPR * u < parts ? a.part[((p0 + WPR * u) * all_rows + row) * D + lane * C + c] : 0.f;
#pragma unroll
    for (int u = 0; u < U; u++) {
      const float fp = __shfl(f, (p0 + WPR * u) & 63);
#pragma unroll
      for (int c = 0; c < C; c++) x[c] = p0 + WPR * u < parts ? __fmaf_rn(fp, y[u][c], x[c]) : x[c];
    }
  }
  E* op = static_cast<E*>(a.out) + (q.off + i) * a.ld_out + head * D;
  if constexpr (WPR == 1) {
#pragma unroll
    for (int c = 0; c < C; c++) op[lane * C + c] = static_cast<E>(x[c] * inv);
  } else {
#pragma unroll
    for (int c = 0; c < C; c++) sums[wave][lane * C + c] = x[c];
    __syncthreads();
    const int c = threadIdx.x;
    if (c < D) op[c] = static_cast<E>((((sums[0][c] + sums[1][c]) + sums[2][c]) + sums[3][c]) * inv);
  }
}

}  // namespace
}  // namespace cache
}  // namespace moe
