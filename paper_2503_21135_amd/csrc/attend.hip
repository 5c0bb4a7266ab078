// attend.hip -- moe_tree_attention: softmax(scale q k) v of drafted tokens over a
// paged cache, each token seeing the cached tokens and the drafts its mask names.
//
// The rows of one matrix tile are the (draft, query head) pairs of one key/value head:
// row r is draft r / G, query head g*G + r % G, so a head's keys are read once for all
// of them.  Both products keep the rows in the lanes of the matrix tile's columns:
//   S^T[key][row] = K Q^T   and   O^T[d][row] += V^T P^T
// so a lane owns one row (lane % 16) of scores, softmax state and outputs, and its
// scores, once exponentiated, already are the second product's operand: tile kt of 16
// keys takes keys 8*(r/4) + 4*kt + r%4 as its row r, which leaves lane group g = lane / 16
// with the keys 8g .. 8g+7 in order.  K rows and (transposed) V rows are read from
// memory straight into operands, 16 bytes a lane, with no pass through LDS.
#include <type_traits>

#include "cache.hpp"

namespace moe {
namespace cache {
namespace {

constexpr int kTile = 32;        // keys of a wave's step; divides every page size
constexpr int kWaves = 4;
constexpr int kMaxSplit = 64;    // the joining wave holds one part's statistics per lane

struct AttendArgs {
  Batch b;
  const void *q, *kc, *vc;
  void* out;
  float *part, *stat;   // [n_split][rows][D] sums and [n_split][rows][2] (maximum, sum) of the parts
  const uint64_t* mask;
  int64_t ld_q, ld_out;
  float scale2;         // scale * log2(e): scores are powers of two
  int n_q_heads, group, mask_words, n_split, row_blocks, rows_wave, units;
};

// Parts of a sequence's keys, in tiles.
__device__ __forceinline__ int tiles_per_part(int tiles, int n_split) { return (tiles + n_split - 1) / n_split; }

template <int TYPE>
__device__ __forceinline__ f32x4 product(const u32x4& a, const u32x4& b, const f32x4& c) {
  if constexpr (TYPE == MOE_TYPE_BF16) return mfma16(a, b, c);
  else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// halves of w that are infinite or NaN, as 0xFFFF each
template <int TYPE>
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
  constexpr uint32_t lo = TYPE == MOE_TYPE_BF16 ? 0x7F80u : 0x7C00u, hi = lo << 16;
  return ((w & lo) == lo ? 0xFFFFu : 0u) | ((w & hi) == hi ? 0xFFFF0000u : 0u);
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

template <int TYPE, int D, int RT>
__global__ void __launch_bounds__(kWaves * kWave, D * RT <= 256 ? 2 : 1) attend_kernel(AttendArgs a) {
  typedef elem_t<TYPE> E;
  constexpr int NC = D / 32, NV = D / 16;
  __shared__ float stats[kWaves][RT][16][2];
  __shared__ float sums[kWaves][16][D + 4];
  // row blocks of a unit (sequence, head, part) sit 8 workgroups apart, on one XCD, and
  // share its keys in that XCD's L2
  const int unit = static_cast<int>(blockIdx.x) / (8 * a.row_blocks) * 8 + static_cast<int>(blockIdx.x) % 8;
  const int rb = static_cast<int>(blockIdx.x) / 8 % a.row_blocks;
  if (unit >= a.units) return;
  const int part = unit % a.n_split, h = unit / a.n_split % a.b.n_heads, s = unit / a.n_split / a.b.n_heads;
  const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = wave % a.rows_wave, wk = wave / a.rows_wave, key_waves = kWaves / a.rows_wave;
  bool ok;
  const Seq q = sequence(a.b, s, ok);
  if (!ok && threadIdx.x == 0) report(a.b, MOE_ERR_SLOT);
  const int rows = q.n * a.group, row0 = rb * a.rows_wave * RT * 16;
  if (row0 >= rows) return;
  const int total = q.len + q.n, tiles = (total + kTile - 1) / kTile, per = tiles_per_part(tiles, a.n_split);
  const int t_end = min(tiles, (part + 1) * per), t_begin = part * per + wk;
  if (part * per >= tiles) return;

  u32x4 qf[RT][NC];
  int tok[RT];      // this lane's row of each row tile: its draft
#pragma unroll
  for (int rt = 0; rt < RT; rt++) {
    const int r = min(row0 + (wr * RT + rt) * 16 + col, rows - 1);
    tok[rt] = r / a.group;
    const E* p = static_cast<const E*>(a.q) + (q.off + tok[rt]) * a.ld_q + (h * a.group + r % a.group) * D + 8 * grp;
#pragma unroll
    for (int c = 0; c < NC; c++) qf[rt][c] = *reinterpret_cast<const u32x4*>(p + 32 * c);
  }
  f32x4 o[RT][NV];
  float m[RT], l[RT];
#pragma unroll
  for (int rt = 0; rt < RT; rt++) {
    m[rt] = -INFINITY;
    l[rt] = 0.f;
#pragma unroll
    for (int v = 0; v < NV; v++) o[rt][v] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  const int P = 1 << a.b.page_shift;
  // pages of this wave's next 64 tiles, one per lane
  int pages = -1;
  auto look_up = [&](int t) {
    const int tl = t + lane * key_waves;
    pages = tl < t_end ? page_of(a.b, s, tl * kTile) : 0;
    if (pages < 0) report(a.b, MOE_ERR_SLOT);
  };
  auto head_at = [&](int page) { return (static_cast<int64_t>(max(page, 0)) * a.b.n_heads + h) * P * D; };
  const int krow = 8 * (col >> 2) + (col & 3);
  auto load_k = [&](u32x4 (&kf)[2][NC], int page, int t) {
    const E* p = static_cast<const E*>(a.kc) + head_at(page);
    const int off = ((t * kTile & (P - 1)) + krow) * D + 8 * grp;
#pragma unroll
    for (int kt = 0; kt < 2; kt++)
#pragma unroll
      for (int c = 0; c < NC; c++) kf[kt][c] = *reinterpret_cast<const u32x4*>(p + off + 4 * kt * D + 32 * c);
  };
  auto load_v = [&](u32x4 (&vf)[NV], int page, int t) {
    const E* p = static_cast<const E*>(a.vc) + head_at(page);
    const int off = col * P + (t * kTile & (P - 1)) + 8 * grp;
#pragma unroll
    for (int v = 0; v < NV; v++) vf[v] = *reinterpret_cast<const u32x4*>(p + off + 16 * v * P);
  };

  // One tile: scores, softmax state, and the second product.  EDGE: slots that not
  // everybody sees are among the tile's (drafts, or none at all).
  auto step = [&](auto edge_c, const u32x4 (&kf)[2][NC], u32x4 (&vf)[NV], int page, int t) {
    constexpr bool EDGE = decltype(edge_c)::value;
    const int j0 = t * kTile + 8 * grp;
    f32x4 sc[RT][2];
#pragma unroll
    for (int rt = 0; rt < RT; rt++)
#pragma unroll
      for (int kt = 0; kt < 2; kt++) {
        f32x4 x = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < NC; c++) x = product<TYPE>(kf[kt][c], qf[rt][c], x);
        sc[rt][kt] = x;
      }
    uint32_t odd = 0;     // this lane's keys with a value that is not finite
    if constexpr (EDGE) {
      const int valid = min(max(total - j0, 0), 8);
      uint32_t in[4];
#pragma unroll
      for (int i = 0; i < 4; i++) in[i] = valid >= 2 * i + 2 ? 0xFFFFFFFFu : (valid == 2 * i + 1 ? 0xFFFFu : 0u);
#pragma unroll
      for (int v = 0; v < NV; v++)
#pragma unroll
        for (int i = 0; i < 4; i++) {
          const uint32_t bad = not_finite<TYPE>(vf[v][i]) & in[i];
          vf[v][i] &= in[i] & ~bad;
          odd |= (bad & 1u) << 2 * i | (bad >> 31) << (2 * i + 1);
        }
    }
    u32x4 pf[RT];
    uint32_t see[RT];
#pragma unroll
    for (int rt = 0; rt < RT; rt++) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; e++) x[e] = sc[rt][e >> 2][e & 3] * a.scale2;
      if constexpr (EDGE) {
        see[rt] = seen8(a, q.off + tok[rt], tok[rt], q.n, j0 - q.len);
#pragma unroll
        for (int e = 0; e < 8; e++) x[e] = see[rt] >> e & 1 ? x[e] : -INFINITY;
      }
      float mx = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
      mx = rows_max(mx);
      const float m2 = fmaxf(m[rt], mx), ms = m2 == -INFINITY ? 0.f : m2;
      if (__any(m2 > m[rt])) {
        const float f = __builtin_amdgcn_exp2f(m[rt] - ms);
        l[rt] *= f;
#pragma unroll
        for (int v = 0; v < NV; v++)
#pragma unroll
          for (int i = 0; i < 4; i++) o[rt][v][i] *= f;
        m[rt] = m2;
      }
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; e++) p[e] = __builtin_amdgcn_exp2f(x[e] - ms);
      l[rt] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
      pf[rt] = u32x4{pack2<TYPE>(p[0], p[1]), pack2<TYPE>(p[2], p[3]), pack2<TYPE>(p[4], p[5]), pack2<TYPE>(p[6], p[7])};
    }
#pragma unroll
    for (int v = 0; v < NV; v++)
#pragma unroll
      for (int rt = 0; rt < RT; rt++) o[rt][v] = product<TYPE>(vf[v], pf[rt], o[rt][v]);
    if constexpr (EDGE) {
      if (!__any(odd != 0)) return;
      // Infinite and NaN values left the product, where 0 * NaN would reach the rows that
      // do not see them; here they go to the rows that do.
      const E* vp = static_cast<const E*>(a.vc) + head_at(page) + (t * kTile & (P - 1)) + 4 * grp * P;
#pragma unroll 1
      for (int key = 0; key < kTile; key++) {
        if (!__any(grp == key >> 3 && (odd >> (key & 7) & 1))) continue;
#pragma unroll
        for (int rt = 0; rt < RT; rt++) {
          uint32_t w = pf[rt][0];
#pragma unroll
          for (int i = 1; i < 4; i++) w = (key & 7) >> 1 == i ? pf[rt][i] : w;
          w = __shfl(w, 16 * (key >> 3) + col);
          const float p = key & 1 ? half_hi<TYPE>(w) : half_lo<TYPE>(w);
          const bool sees = __shfl(see[rt], 16 * (key >> 3) + col) >> (key & 7) & 1;
#pragma unroll
          for (int v = 0; v < NV; v++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
              const float x = static_cast<float>(vp[(16 * v + i) * P + key]);
              o[rt][v][i] += __builtin_isfinite(x) || !sees ? 0.f : p * x;
            }
        }
      }
    }
  };

  // Tiles whose slots all hold cached tokens come first, the next tile's keys loading
  // behind this one's products; the last ones, with drafts in them, one at a time.
  const int t_full = min(t_end, q.len / kTile);
  int left = 0, t = t_begin;
  if (t < t_end) look_up(t);
  if (t < t_full) {
    u32x4 kf[2][NC], vf[NV], kn[2][NC];
    int page = __builtin_amdgcn_readfirstlane(pages);
    load_k(kf, page, t);
    for (; t < t_full; t += key_waves) {
      load_v(vf, page, t);
      if (++left == kWave) {
        look_up(t + key_waves);
        left = 0;
      }
      const int next = __builtin_amdgcn_readlane(pages, left);
      if (t + key_waves < t_full) load_k(kn, next, t + key_waves);
      if (page >= 0) step(std::false_type{}, kf, vf, page, t);
#pragma unroll
      for (int kt = 0; kt < 2; kt++)
#pragma unroll
        for (int c = 0; c < NC; c++) kf[kt][c] = kn[kt][c];
      page = next;
    }
  }
#pragma unroll 1
  for (; t < t_end; t += key_waves) {
    const int page = __builtin_amdgcn_readlane(pages, left);
    if (page >= 0) {
      u32x4 kf[2][NC], vf[NV];
      load_k(kf, page, t);
      load_v(vf, page, t);
      step(std::true_type{}, kf, vf, page, t);
    }
    if (++left == kWave) {
      look_up(t + key_waves);
      left = 0;
    }
  }

  // join the waves that shared the rows: common maximum, then the sums in wave order
#pragma unroll
  for (int rt = 0; rt < RT; rt++) {
    l[rt] = rows_sum(l[rt]);
    if (grp == 0) {
      stats[wave][rt][col][0] = m[rt];
      stats[wave][rt][col][1] = l[rt];
    }
  }
  __syncthreads();
  const int64_t all_rows = static_cast<int64_t>(a.b.n_seqs) * a.b.max_new * a.n_q_heads;
#pragma unroll
  for (int rt = 0; rt < RT; rt++) {
    float top = -INFINITY;
    for (int w = 0; w < key_waves; w++) top = fmaxf(top, stats[w * a.rows_wave + wr][rt][col][0]);
    const float f = m[rt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[rt] - top);
    if (rt) __syncthreads();
#pragma unroll
    for (int v = 0; v < NV; v++) {
      f32x4 x = o[rt][v];
#pragma unroll
      for (int i = 0; i < 4; i++) x[i] *= f;
      *reinterpret_cast<f32x4*>(&sums[wave][col][16 * v + 4 * grp]) = x;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.rows_wave * 16 * (D / 4); i += kWaves * kWave) {
      const int c = i % (D / 4) * 4, rr = i / (D / 4) % 16, w0 = i / (D / 4) / 16;
      const int r = row0 + (w0 * RT + rt) * 16 + rr;
      if (r >= rows) continue;
      float hi = -INFINITY, sum = 0.f;
      for (int w = 0; w < key_waves; w++) hi = fmaxf(hi, stats[w * a.rows_wave + w0][rt][rr][0]);
      f32x4 x = f32x4{0.f, 0.f, 0.f, 0.f};
      for (int w = 0; w < key_waves; w++) {
        const float mw = stats[w * a.rows_wave + w0][rt][rr][0];
        if (mw != -INFINITY) sum += stats[w * a.rows_wave + w0][rt][rr][1] * __builtin_amdgcn_exp2f(mw - hi);
        const f32x4 y = *reinterpret_cast<const f32x4*>(&sums[w * a.rows_wave + w0][rr][c]);
#pragma unroll
        for (int e = 0; e < 4; e++) x[e] += y[e];
      }
      const int i_tok = r / a.group, head = h * a.group + r % a.group;
      if (a.n_split == 1) {
        const float inv = sum == 0.f ? 0.f : 1.0f / sum;
        E* op = static_cast<E*>(a.out) + (q.off + i_tok) * a.ld_out + head * D + c;
#pragma unroll
        for (int e = 0; e < 4; e++) op[e] = static_cast<E>(x[e] * inv);
      } else {
        const int64_t row = part * all_rows + (static_cast<int64_t>(s) * a.b.max_new + i_tok) * a.n_q_heads + head;
        *reinterpret_cast<f32x4*>(a.part + row * D + c) = x;
        if (c == 0) {
          a.stat[2 * row] = hi;
          a.stat[2 * row + 1] = sum;
        }
      }
    }
  }
}

// One wave per (new token, query head): joins its parts in order.
template <int TYPE, int D>
__global__ void __launch_bounds__(256) join_kernel(AttendArgs a) {
  typedef elem_t<TYPE> E;
  const int64_t all_rows = static_cast<int64_t>(a.b.n_seqs) * a.b.max_new * a.n_q_heads;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (row >= all_rows) return;
  const int head = static_cast<int>(row % a.n_q_heads);
  const int64_t tok = row / a.n_q_heads;
  const int s = static_cast<int>(tok / a.b.max_new), i = static_cast<int>(tok % a.b.max_new);
  bool ok;
  const Seq q = sequence(a.b, s, ok);
  if (i >= q.n) return;
  const int tiles = (q.len + q.n + kTile - 1) / kTile, per = tiles_per_part(tiles, a.n_split);
  const int parts = (tiles + per - 1) / per;
  float m = -INFINITY, l = 0.f;
  if (lane < parts) {
    m = a.stat[2 * (lane * all_rows + row)];
    l = a.stat[2 * (lane * all_rows + row) + 1];
  }
  float top = m;
  for (int w = 32; w; w >>= 1) top = fmaxf(top, __shfl_xor(top, w));
  const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
  float sum = l * f;
  for (int w = 32; w; w >>= 1) sum += __shfl_xor(sum, w);
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
  float x[D / kWave];
#pragma unroll
  for (int c = 0; c < D / kWave; c++) x[c] = 0.f;
  for (int p = 0; p < parts; p++) {
    const float fp = __shfl(f, p);
#pragma unroll
    for (int c = 0; c < D / kWave; c++) x[c] = __fmaf_rn(fp, a.part[(p * all_rows + row) * D + lane * (D / kWave) + c], x[c]);
  }
  E* op = static_cast<E*>(a.out) + (q.off + i) * a.ld_out + head * D + lane * (D / kWave);
#pragma unroll
  for (int c = 0; c < D / kWave; c++) op[c] = static_cast<E>(x[c] * inv);
}

// How a batch is laid over workgroups.
struct Plan {
  int row_tiles;   // 16-row tiles of a wave
  int rows_wave;   // waves of a workgroup that take other rows; the rest take other keys
  int row_blocks;  // workgroups over the rows
  int n_split;     // parts of the keys
};

Plan plan_of(const moe_cache_t* C, int n_q_heads, int n_seqs, int max_new, int max_len) {
  const int64_t rows = static_cast<int64_t>(max_new) * (n_q_heads / C->n_heads);
  Plan p;
  p.row_tiles = rows <= 16 ? 1 : (rows <= 32 || C->head_dim == 256 ? 2 : 4);
  p.rows_wave = 1;
  while (p.rows_wave < kWaves && p.rows_wave * p.row_tiles * 16 < rows) p.rows_wave *= 2;
  p.row_blocks = static_cast<int>(cdiv(rows, p.rows_wave * p.row_tiles * 16));
  const int64_t wgs = static_cast<int64_t>(n_seqs) * C->n_heads * p.row_blocks;
  const int64_t steps = cdiv(max_len, kTile * (kWaves / p.rows_wave));
  p.n_split = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({cdiv(1024, std::max<int64_t>(wgs, 1)), steps / 2, kMaxSplit})));
  return p;
}

template <int TYPE, int D>
void launch(const Plan& p, hipStream_t s, const AttendArgs& a) {
  const dim3 grid(static_cast<unsigned>(cdiv(a.units, 8) * 8 * p.row_blocks)), block(kWaves * kWave);
  if (p.row_tiles == 1) hipLaunchKernelGGL((attend_kernel<TYPE, D, 1>), grid, block, 0, s, a);
  else if (p.row_tiles == 2) hipLaunchKernelGGL((attend_kernel<TYPE, D, 2>), grid, block, 0, s, a);
  else if constexpr (D < 256) hipLaunchKernelGGL((attend_kernel<TYPE, D, 4>), grid, block, 0, s, a);
  if (p.n_split > 1) {
    const int64_t rows = static_cast<int64_t>(a.b.n_seqs) * a.b.max_new * a.n_q_heads;
    hipLaunchKernelGGL((join_kernel<TYPE, D>), dim3(static_cast<unsigned>(cdiv(rows, 4))), dim3(256), 0, s, a);
  }
}

template <int TYPE>
void launch(int head_dim, const Plan& p, hipStream_t s, const AttendArgs& a) {
  if (head_dim == 64) launch<TYPE, 64>(p, s, a);
  else if (head_dim == 128) launch<TYPE, 128>(p, s, a);
  else launch<TYPE, 256>(p, s, a);
}

int check_sizes(const moe_cache_t* C, int32_t n_q_heads, int32_t n_seqs, int32_t max_new, int32_t max_len) {
  if (int st = check_cache(C)) return st;
  if (n_seqs < 0 || n_seqs > 65535 || max_new < 0 || max_len < 0) return MOE_ERR_ARG;
  if (n_q_heads < 1 || n_q_heads % C->n_heads || n_q_heads / C->n_heads > 64) return MOE_ERR_ARG;
  // rows and workgroups are counted in 31 bits
  if (static_cast<int64_t>(n_seqs) * max_new * n_q_heads > INT32_MAX / kMaxSplit) return MOE_ERR_ARG;
  return MOE_OK;
}

}  // namespace
}  // namespace cache
}  // namespace moe

extern "C" int moe_tree_attention_plan(const moe_cache_t* C, int32_t n_q_heads, int32_t n_seqs,
                                       int32_t max_new, int32_t max_len, int32_t* n_split,
                                       size_t* ws_bytes) {
  using namespace moe::cache;
  if (int st = check_sizes(C, n_q_heads, n_seqs, max_new, max_len)) return st;
  const int n = plan_of(C, n_q_heads, n_seqs, max_new, max_len).n_split;
  if (n_split) *n_split = n;
  if (ws_bytes)
    *ws_bytes = n == 1 ? 0 : sizeof(float) * n * (C->head_dim + 2) * static_cast<size_t>(n_seqs) * max_new * n_q_heads;
  return MOE_OK;
}

extern "C" int moe_tree_attention(const moe_cache_t* C, const int32_t* table, int32_t max_pages,
                                  const int32_t* cache_len, int32_t n_seqs, const int32_t* new_off,
                                  int32_t n_tokens, int32_t max_new, int32_t max_len, const void* q,
                                  int64_t ld_q, int32_t n_q_heads, const uint64_t* mask,
                                  int32_t mask_words, float scale, void* out, int64_t ld_out,
                                  int32_t* status, void* ws, size_t ws_bytes, void* stream) {
  using namespace moe;
  using namespace moe::cache;
  if (int st = check_sizes(C, n_q_heads, n_seqs, max_new, max_len)) return st;
  if (n_tokens < 0 || !__builtin_isfinite(scale) || (mask && mask_words < 1)) return MOE_ERR_ARG;
  if (n_seqs == 0 || n_tokens == 0 || max_new == 0) return MOE_OK;
  if (int st = check_batch(C, table, max_pages, cache_len, new_off)) return st;
  const int64_t width = static_cast<int64_t>(n_q_heads) * C->head_dim;
  if (!q || !out || ld_q < width || ld_out < width) return MOE_ERR_ARG;
  if (!aligned16(q) || ld_q % 8 || !aligned_to(out, 2) || !aligned_to(mask, 8)) return MOE_ERR_ALIGN;
  size_t need = 0;
  if (int st = moe_tree_attention_plan(C, n_q_heads, n_seqs, max_new, max_len, nullptr, &need)) return st;
  if (need > 0 && (!ws || ws_bytes < need)) return MOE_ERR_WORKSPACE;
  if (need > 0 && !aligned16(ws)) return MOE_ERR_ALIGN;
  const Plan p = plan_of(C, n_q_heads, n_seqs, max_new, max_len);
  const int64_t all_rows = static_cast<int64_t>(n_seqs) * max_new * n_q_heads;
  float* part = static_cast<float*>(ws);
  const AttendArgs a{batch_of(C, table, max_pages, cache_len, n_seqs, new_off, n_tokens, max_new, status),
                     q, C->k, C->v, out, part, part + p.n_split * all_rows * C->head_dim, mask, ld_q, ld_out,
                     scale * 1.44269504088896340736f, n_q_heads, n_q_heads / C->n_heads, mask_words, p.n_split,
                     p.row_blocks, p.rows_wave, n_seqs * C->n_heads * p.n_split};
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (C->type == MOE_TYPE_BF16) launch<MOE_TYPE_BF16>(C->head_dim, p, s, a);
  else launch<MOE_TYPE_FP16>(C->head_dim, p, s, a);
  return launch_status(s);
}
