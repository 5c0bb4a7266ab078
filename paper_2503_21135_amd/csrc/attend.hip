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
#include <algorithm>
#include <type_traits>

#include "cache.hpp"

namespace moe {
namespace cache {
namespace {

constexpr int kTile = 32;        // keys of a step; divides every page size
// A row's weights are 2^(score - maximum + kLift), with a maximum that may lag 2^kSlack behind.
// In fp16 the lift of 7 keeps the largest finite (2^15) and gives weights that are small beside it
// their place: normal down to 2^-21 of the maximum, zero only below 2^-32 (unlifted, a million
// keys of 2^-26 each, 1.6 % of the sum, counted for nothing).  bf16 has fp32's range.
constexpr float kSlack = 8.f;
template <int TYPE> constexpr float kLift = TYPE == MOE_TYPE_FP16 ? 7.f : 0.f;
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

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// Two weights rounded to a 16-bit type toward zero and one unit further, 0 staying 0: what is
// left over is positive wherever the weight is, so that neither of the two products of an
// infinite value has another sign or is NaN.
template <int TYPE>
__device__ __forceinline__ uint32_t below2(float a, float b) {
  uint32_t w;
  if constexpr (TYPE == MOE_TYPE_BF16) w = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
  else w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(a, b));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_sub_sat(__builtin_bit_cast(u16x2, w), u16x2{1, 1}));
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

// RW = 1: four waves on the same 16 RT rows, each with keys of its own, operands straight
// from memory.  RW > 1: eight waves, RW of them on other rows; those read tiles of keys
// once, side by side, into LDS, and take their operands from there (double-buffered, one
// barrier a stage).  Straight from memory an operand has 16 rows side by side, whose
// 16-byte pieces the vector memory path serves one per cycle: enough for one wave per tile
// to keep up with HBM, not for several on the same one (64 drafts by 4 heads per key head
// over 4 x 32768 slots: 448 us that way, 156 this way, the join included).
//
// Few rows are bound by HBM: 64 sequences of one token over up to 4096, 778 MB, 155 us and
// 4.8 to join, 5.0 TB/s.  At 256 rows per key head (4 x 64 drafts over up to 32768, 88 GFLOP,
// 418 MB: 148 us and 7.8 to join; 193 and 9 on a card that has rested) a tile's matrix
// instructions (1024 cycles of each SIMD), vector instructions (1100) and LDS reads (1150)
// follow each other rather than overlap: matrix instructions fill 39 % of a busy CU's
// cycles.  And parts are uneven: of lengths from 18706 to 32768 they make 208 workgroups
// of up to 129 tiles, where an even share of 256 CUs is 99, and parts of one number fall on
// one XCD.  Giving one wave of a SIMD the higher priority, or the waves in their matrix
// instructions, left that as it was, and so did reading the value operands before the softmax.
template <int TYPE, int D, int RT, int RW>
__global__ void __launch_bounds__(RW == 1 ? 256 : 512, D <= 128 || RW > 1 ? 2 : 1) attend_kernel(AttendArgs a) {
  typedef elem_t<TYPE> E;
  constexpr int NC = D / 32, NV = D / 16, W = RW == 1 ? 4 : 8, KW = W / RW;
  // The second product takes weights as operands of the cache's type.  Few rows, which wait for
  // HBM, add the product with what a rounding down left over, so that the output's error is its own
  // rounding's (64 x 1 over 4096, bf16: 1.7e-3 against 64 bits, else 2.3e-3) at the same time
  // (160.1 us both ways; 64 x 8 drafts of head_dim 64 over 2000 58.3 instead of 57.8).  Many rows would
  // pay for it: 4 x 64 over 32768 206 us instead of 156, 8 x 32 over 8000 79 instead of 71.
  constexpr bool kRest = RW == 1;
  // tiles that a key group stages at once (4 x 64 over 32768: one 159 us, two 161, four 169;
  // head_dim 64 over 8000: two 39, four 42, and one would leave threads without a piece),
  // threads of a key group, and their 16-byte pieces of a stage's keys
  constexpr int KT = RW == 1 ? 1 : std::min(2, RW * 64 / D), TG = RW * kWave, NP = KT * 4 * D / TG;
  struct Tile {
    u32x4 k[kTile][D / 8];    // row 16 kt + col is the operand row of lane col in tile kt; pieces and rows are
    u32x4 v[D][kTile / 8];    // mixed so that 16 lanes' reads fall on all banks
  };
  struct Sums { float x[W][16][D + 4]; };
  union Lds {
    Tile tile[2][KW][KT];
    Sums sums;
  };
  __shared__ __attribute__((aligned(16))) char lds_bytes[RW == 1 ? sizeof(Sums) : sizeof(Lds)];
  __shared__ float stats[W][RT][16][2];
  // row blocks of a unit (sequence, head, part) sit 8 workgroups apart, on one XCD, and
  // share its keys in that XCD's L2
  const int unit = static_cast<int>(blockIdx.x) / (8 * a.row_blocks) * 8 + static_cast<int>(blockIdx.x) % 8;
  const int rb = static_cast<int>(blockIdx.x) / 8 % a.row_blocks;
  if (unit >= a.units) return;
  const int part = unit % a.n_split, h = unit / a.n_split % a.b.n_heads, s = unit / a.n_split / a.b.n_heads;
  const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = wave % RW, wk = wave / RW;
  bool ok;
  const Seq q = sequence(a.b, s, ok);
  if (!ok && threadIdx.x == 0) report(a.b, MOE_ERR_SLOT);
  const int rows = q.n * a.group, row0 = rb * RW * RT * 16;
  if (row0 >= rows) return;
  const int total = q.len + q.n, tiles = (total + kTile - 1) / kTile, per = tiles_per_part(a, tiles);
  if (static_cast<int64_t>(part) * per >= tiles) return;
  const int t_first = part * per, t_end = per >= tiles - t_first ? tiles : t_first + per;

  u32x4 qf[RT][NC];
  int tok[RT];      // this lane's row of each row tile: its draft
#pragma unroll
  for (int rt = 0; rt < RT; rt++) {
    const int r = min(row0 + (wr * RT + rt) * 16 + col, rows - 1);   // a row past the last is its copy, not stored
    tok[rt] = r / a.group;
    const E* p = static_cast<const E*>(a.q) + (q.off + tok[rt]) * a.ld_q + (h * a.group + r % a.group) * D + 8 * grp;
#pragma unroll
    for (int c = 0; c < NC; c++) qf[rt][c] = *reinterpret_cast<const u32x4*>(p + 32 * c) ^ u32x4{a.flip, a.flip, a.flip, a.flip};
  }
  f32x4 o[RT][NV];
  float m[RT], ms[RT], l[RT];   // maximum, the same scaled less the lift, sum
#pragma unroll
  for (int rt = 0; rt < RT; rt++) {
    m[rt] = ms[rt] = -INFINITY;
    l[rt] = 0.f;
#pragma unroll
    for (int v = 0; v < NV; v++) o[rt][v] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  const int P = 1 << a.b.page_shift;
  // this wave's n-th tile, and the pages of 64 of them from the n-th on, one per lane
  auto tile_of = [&](int n) { return t_first + (n / KT * KW + wk) * KT + n % KT; };
  int pages = -1;
  auto look_up = [&](int n) {
    const int tl = tile_of(n + lane);
    pages = tl < t_end ? page_of(a.b, s, tl * kTile) : 0;
    if (pages < 0) report(a.b, MOE_ERR_SLOT);
  };
  auto head_at = [&](int page) { return (static_cast<int64_t>(max(page, 0)) * a.b.n_heads + h) * P * D; };
  const int krow = 8 * (col >> 2) + (col & 3);
  // a uniform base and a 32-bit offset per lane
  const uint32_t k_off = krow * D + 8 * grp, v_off = col * P + 8 * grp, o_off = 4 * grp * P;
  auto load_k = [&](u32x4 (&kf)[2][NC], int page, int t) {
    const E* p = static_cast<const E*>(a.kc) + head_at(page) + (t * kTile & (P - 1)) * D;
#pragma unroll
    for (int kt = 0; kt < 2; kt++)
#pragma unroll
      for (int c = 0; c < NC; c++) kf[kt][c] = *reinterpret_cast<const u32x4*>(p + (k_off + 4 * kt * D + 32 * c));
  };
  auto load_v = [&](u32x4 (&vf)[NV], int page, int t) {
    const E* p = static_cast<const E*>(a.vc) + head_at(page) + (t * kTile & (P - 1));
#pragma unroll
    for (int v = 0; v < NV; v++) vf[v] = *reinterpret_cast<const u32x4*>(p + 16 * v * P + v_off);
  };

  const int t_full = min(t_end, q.len / kTile);    // tiles before it hold cached tokens alone
  uint32_t odd = 0;   // not 0: this wave left values out that are not finite
  // One tile: scores, softmax state, and the second product.  EDGE: slots that not
  // everybody sees (drafts, or none at all) may be among the tile's, and are from t_full on.
  // get_k and get_v give the tile's operands, from registers or LDS.
  auto step = [&](auto edge_c, auto get_k, auto get_v, int t) {
    constexpr bool EDGE = decltype(edge_c)::value;
    const int j0 = t * kTile + 8 * grp;
    f32x4 sc[RT][2];
#pragma unroll
    for (int kt = 0; kt < 2; kt++)
#pragma unroll
      for (int c = 0; c < NC; c++) {
        const u32x4 k = get_k(kt, c);
#pragma unroll
        for (int rt = 0; rt < RT; rt++) sc[rt][kt] = product<TYPE>(k, qf[rt][c], c ? sc[rt][kt] : f32x4{0.f, 0.f, 0.f, 0.f});
      }
    u32x4 pf[RT], rest[RT];
#pragma unroll
    for (int rt = 0; rt < RT; rt++) {
      float x[8], y[8];
      uint32_t see = 0xFFu;
      if constexpr (EDGE) see = seen8(a, q.off + tok[rt], tok[rt], q.n, j0 - q.len);
#pragma unroll
      for (int e = 0; e < 8; e++) {
        x[e] = sc[rt][e >> 2][e & 3];
        if constexpr (EDGE) x[e] = see >> e & 1 ? x[e] : -INFINITY;
        y[e] = __fmaf_rn(x[e], a.scale2, -ms[rt]);
      }
      auto most = [](const float (&v)[8]) {
        return fmaxf(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7])));
      };
      // A row's maximum moves only when a score passes it by kSlack: until then weights
      // stay below 2^(kSlack + kLift), and no lane asks the others for theirs.  (A row that has seen
      // nothing has -infinity, which any score passes.)
      if (__any(!(most(y) <= kSlack + kLift<TYPE>))) {
        const bool moves = !(rows_max(most(y)) <= kSlack + kLift<TYPE>);    // this row, whatever its neighbours do
        const float m2 = moves ? fmaxf(m[rt], rows_max(most(x))) : m[rt];
        const float ms2 = m2 == -INFINITY ? 0.f : m2 * a.scale2 - kLift<TYPE>;
        const float f = m[rt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ms[rt] - ms2);
        l[rt] *= f;
#pragma unroll
        for (int v = 0; v < NV; v++)
#pragma unroll
          for (int i = 0; i < 4; i++) o[rt][v][i] *= f;
        m[rt] = m2;
        ms[rt] = m2 == -INFINITY ? -INFINITY : ms2;
#pragma unroll
        for (int e = 0; e < 8; e++) y[e] = __fmaf_rn(x[e], a.scale2, -ms2);
      }
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; e++) {
        p[e] = __builtin_amdgcn_exp2f(y[e]);
        if constexpr (EDGE) p[e] = see >> e & 1 ? p[e] : 0.f;
      }
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const float a = p[2 * i], b = p[2 * i + 1];
        pf[rt][i] = kRest ? below2<TYPE>(a, b) : pack2<TYPE>(a, b);
        if constexpr (kRest) rest[rt][i] = pack2<TYPE>(a - half_lo<TYPE>(pf[rt][i]), b - half_hi<TYPE>(pf[rt][i]));
      }
      // the sum is that of the rounded weights, so that what rounding does to a weight that
      // outweighs the rest cancels
#pragma unroll
      for (int i = 0; i < 4; i++) {
        l[rt] = dot2<TYPE>(pf[rt][i], kOnes<TYPE>, l[rt]);
        if constexpr (kRest) l[rt] = dot2<TYPE>(rest[rt][i], kOnes<TYPE>, l[rt]);
      }
    }
    const int valid = min(max(total - j0, 0), 8);
    const uint32_t scrub = RW > 1 && t < t_full ? 0u : 0xFFFFFFFFu;   // a stage's edge may be behind this tile of it
#pragma unroll
    for (int v = 0; v < NV; v++) {
      u32x4 w = get_v(v);
      if constexpr (EDGE)
#pragma unroll
        for (int i = 0; i < 4; i++) {   // slots past the last token, and what is not finite but not seen by all, as zeros
          const uint32_t in = valid >= 2 * i + 2 ? 0xFFFFFFFFu : (valid == 2 * i + 1 ? 0xFFFFu : 0u);
          const uint32_t bad = not_finite<TYPE>(w[i]) & in & scrub;
          w[i] &= in & ~bad;
          odd |= bad;
        }
#pragma unroll
      for (int rt = 0; rt < RT; rt++) {
        o[rt][v] = product<TYPE>(w, pf[rt], o[rt][v]);
        if constexpr (kRest) o[rt][v] = product<TYPE>(w, rest[rt], o[rt][v]);
      }
    }
  };

  if constexpr (RW == 1) {
    // the next tile's keys load behind this one's products; tiles with drafts in them, the
    // last ones, go one at a time
    int n = 0, t = t_first + wk;
    auto next_page = [&]() {
      if (++n % kWave == 0) look_up(n);
      return static_cast<int>(__builtin_amdgcn_readlane(pages, n % kWave));
    };
    look_up(0);
    int page = __builtin_amdgcn_readfirstlane(pages);
    if (t < t_full) {
      u32x4 kf[2][NC], vf[NV], kn[2][NC];
      load_k(kf, page, t);
      for (; t < t_full; t += KW) {
        load_v(vf, page, t);
        const int next = next_page();
        if (t + KW < t_full) load_k(kn, next, t + KW);
        if (page >= 0)
          step(std::false_type{}, [&](int kt, int c) { return kf[kt][c]; }, [&](int v) { return vf[v]; }, t);
#pragma unroll
        for (int kt = 0; kt < 2; kt++)
#pragma unroll
          for (int c = 0; c < NC; c++) kf[kt][c] = kn[kt][c];
        page = next;
      }
    }
#pragma unroll 1
    for (; t < t_end; t += KW) {
      if (page >= 0) {
        u32x4 kf[2][NC], vf[NV];
        load_k(kf, page, t);
        load_v(vf, page, t);
        step(std::true_type{}, [&](int kt, int c) { return kf[kt][c]; }, [&](int v) { return vf[v]; }, t);
      }
      page = next_page();
    }
  } else {
    Lds& lds = *reinterpret_cast<Lds*>(lds_bytes);
    const int tid = threadIdx.x % TG, wtid = wr * kWave;
    u32x4 kp[NP], vp[NP];
    // loads of stage r; bit j of the answer: its j-th tile is there
    auto load = [&](int r) {
      if (r * KT % kWave == 0) look_up(r * KT);
      uint32_t there = 0;
#pragma unroll
      for (int j = 0; j < KT; j++) {
        const int t = tile_of(r * KT + j), page = __builtin_amdgcn_readlane(pages, (r * KT + j) % kWave);
        if (t >= t_end || page < 0) continue;
        there |= 1u << j;
        const E *kb = static_cast<const E*>(a.kc) + head_at(page) + (t * kTile & (P - 1)) * D;
        const E *vb = static_cast<const E*>(a.vc) + head_at(page) + (t * kTile & (P - 1));
#pragma unroll
        for (int i = 0; i < NP; i++) {
          if ((wtid + i * TG) / (4 * D) != j) continue;     // the same for a whole wave
          const uint32_t x = (tid + i * TG) % (4 * D);
          kp[i] = *reinterpret_cast<const u32x4*>(kb + x * 8);
          vp[i] = *reinterpret_cast<const u32x4*>(vb + ((x >> 2) * P + (x & 3) * 8));
        }
      }
      return there;
    };
    uint32_t there = load(0);
    auto stage = [&](auto edge_c, int r) {
      Tile (&tiles_r)[KT] = lds.tile[r & 1][wk];
#pragma unroll
      for (int i = 0; i < NP; i++) {
        Tile& tile = tiles_r[(wtid + i * TG) / (4 * D)];
        const int x = (tid + i * TG) % (4 * D), key = x / (D / 8), row = 16 * (key >> 2 & 1) + 4 * (key >> 3) + (key & 3);
        tile.k[row][x % (D / 8) ^ (D == 64 ? row >> 1 & 7 : row & 15)] = kp[i];
        tile.v[x >> 2][(x & 3) ^ (x >> 4 & 3)] = vp[i];
      }
      const uint32_t now = there;
      __syncthreads();
      there = load(r + 1);
#pragma unroll 1
      for (int j = 0; j < KT; j++) {
        const Tile& tile = tiles_r[j];
        if (now >> j & 1)
          step(edge_c, [&](int kt, int c) { return tile.k[16 * kt + col][(4 * c + grp) ^ (D == 64 ? col >> 1 : col)]; },
               [&](int v) { return tile.v[16 * v + col][grp ^ (col >> 2)]; }, tile_of(r * KT + j));
      }
    };
    const int stages = (t_end - t_first + KW * KT - 1) / (KW * KT), full = max(0, t_full - t_first) / (KW * KT);
    for (int r = 0; r < full; r++) stage(std::false_type{}, r);
#pragma unroll 1
    for (int r = full; r < stages; r++) stage(std::true_type{}, r);
    __syncthreads();    // the tiles' place is taken by the sums
  }

  if (__any(odd != 0)) {
    // Infinite and NaN values of tiles from t_full on were left out of the products, where 0 * NaN
    // would have reached the rows that do not see them; here they go to the rows that do.
#pragma unroll 1
    for (int n = 0; n < (t_end - t_first + KW * KT - 1) / (KW * KT) * KT; n++) {
      const int tf = tile_of(n);
      if (tf < t_full || tf >= t_end) continue;
      const int pg = __builtin_amdgcn_readfirstlane(page_of(a.b, s, tf * kTile));
      if (pg < 0) continue;
      const E* kb = static_cast<const E*>(a.kc) + head_at(pg) + (tf * kTile & (P - 1)) * D;
      const E* vb = static_cast<const E*>(a.vc) + head_at(pg) + (tf * kTile & (P - 1));
#pragma unroll
      for (int rt = 0; rt < RT; rt++)
#pragma unroll 1
        for (int key = 0; key < min(kTile, total - tf * kTile); key++) {
          // the score of this lane's row and the key, from the four lanes that hold the row
          float x = 0.f;
#pragma unroll 1
          for (int c = 0; c < NC; c++) {
            u32x4 qc = qf[rt][0];
#pragma unroll
            for (int i = 1; i < NC; i++) qc = c == i ? qf[rt][i] : qc;
            const u32x4 k = *reinterpret_cast<const u32x4*>(kb + key * D + 32 * c + 8 * grp);
#pragma unroll
            for (int i = 0; i < 4; i++)
              x += half_lo<TYPE>(qc[i]) * half_lo<TYPE>(k[i]) + half_hi<TYPE>(qc[i]) * half_hi<TYPE>(k[i]);
          }
          x = rows_sum(x);
          const bool sees = seen8(a, q.off + tok[rt], tok[rt], q.n, tf * kTile + key - q.len) & 1;
          const float p = __builtin_amdgcn_exp2f(__fmaf_rn(x, a.scale2, m[rt] == -INFINITY ? 0.f : -ms[rt]));
#pragma unroll
          for (int v = 0; v < NV; v++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
              const float val = static_cast<float>((vb + key + (16 * v + i) * P)[o_off]);
              if (!__builtin_isfinite(val) && sees) o[rt][v][i] += p * val;
              __builtin_amdgcn_sched_barrier(0);   // one load at a time: registers for a rare case
            }
        }
    }
  }
  Sums& sums = *reinterpret_cast<Sums*>(lds_bytes);

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
    for (int w = 0; w < KW; w++) top = fmaxf(top, stats[w * RW + wr][rt][col][0]);
    const float f = m[rt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m[rt] - top) * a.scale2);
    if (rt) __syncthreads();
#pragma unroll
    for (int v = 0; v < NV; v++) {
      f32x4 x = o[rt][v];
#pragma unroll
      for (int i = 0; i < 4; i++) x[i] *= f;
      *reinterpret_cast<f32x4*>(&sums.x[wave][col][16 * v + 4 * grp]) = x;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < RW * 16 * (D / 4); i += W * kWave) {
      const int c = i % (D / 4) * 4, rr = i / (D / 4) % 16, w0 = i / (D / 4) / 16;
      const int r = row0 + (w0 * RT + rt) * 16 + rr;
      if (r >= rows) continue;
      float hi = -INFINITY, sum = 0.f;
      for (int w = 0; w < KW; w++) hi = fmaxf(hi, stats[w * RW + w0][rt][rr][0]);
      f32x4 x = f32x4{0.f, 0.f, 0.f, 0.f};
      for (int w = 0; w < KW; w++) {
        const float mw = stats[w * RW + w0][rt][rr][0];
        if (mw != -INFINITY) sum += stats[w * RW + w0][rt][rr][1] * __builtin_amdgcn_exp2f((mw - hi) * a.scale2);
        const f32x4 y = *reinterpret_cast<const f32x4*>(&sums.x[w * RW + w0][rr][c]);
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

// Joins the parts of each (new token, query head): WPR waves take every WPR-th part, lanes
// side by side over the channels, and are added in wave order.
template <int TYPE, int D, int WPR>
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
  const int tiles = (q.len + q.n + kTile - 1) / kTile, per = tiles_per_part(a, tiles);
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

// How a batch is laid over workgroups.  Up to 16 rows (32 where the registers allow two
// tiles) per key head go straight from memory, more through LDS with as many row waves as
// it takes.  Parts: enough for 1024 workgroups straight from memory (four a CU), 256 through LDS
// (one a CU; with 512, which run one after another, the large trees take 176 us instead
// of 160, 2 x 32 drafts over 16000 60 instead of 47, 4 x 12 of head_dim 256 over 4000 36
// instead of 26, joins included), and no shorter than two steps of every wave.
struct Plan {
  int row_waves;   // RW of the kernel
  int row_tiles;   // 16-row tiles of a wave
  int row_blocks;  // workgroups over the rows
  int n_split;     // parts of the keys
  int part_tiles;  // tiles of a part of the longest sequence
};

Plan plan_of(const moe_cache_t* C, int n_q_heads, int n_seqs, int max_new, int max_len) {
  const int64_t rows = static_cast<int64_t>(max_new) * (n_q_heads / C->n_heads);
  const bool wide = C->head_dim == 256;
  Plan p;
  p.row_tiles = wide || rows <= 16 ? 1 : 2;
  p.row_waves = 1;
  if (rows > 16 * p.row_tiles)
    for (p.row_waves = wide ? 4 : 2; p.row_waves < 8 && p.row_waves * p.row_tiles * 16 < rows;) p.row_waves *= 2;
  p.row_blocks = static_cast<int>(cdiv(rows, p.row_waves * p.row_tiles * 16));
  const int key_waves = (p.row_waves == 1 ? 4 : 8) / p.row_waves;
  const int64_t wgs = std::max<int64_t>(1, static_cast<int64_t>(n_seqs) * C->n_heads * p.row_blocks);
  const int64_t tiles = std::max<int64_t>(1, cdiv(max_len, kTile));
  const int64_t want = std::max<int64_t>(1, std::min<int64_t>({cdiv(p.row_waves == 1 ? 1024 : 256, wgs), tiles / (2 * key_waves), kMaxSplit}));
  p.part_tiles = static_cast<int>(cdiv(tiles, want));
  p.n_split = static_cast<int>(cdiv(tiles, p.part_tiles));
  return p;
}

template <int TYPE, int D>
void launch(const Plan& p, hipStream_t s, const AttendArgs& a) {
  const dim3 grid(static_cast<unsigned>(cdiv(a.units, 8) * 8 * p.row_blocks));
  constexpr int RT = D == 256 ? 1 : 2;
  if (p.row_waves == 1 && p.row_tiles == 1) hipLaunchKernelGGL((attend_kernel<TYPE, D, 1, 1>), grid, dim3(256), 0, s, a);
  else if (p.row_waves == 4) hipLaunchKernelGGL((attend_kernel<TYPE, D, RT, 4>), grid, dim3(512), 0, s, a);
  else if (p.row_waves == 8) hipLaunchKernelGGL((attend_kernel<TYPE, D, RT, 8>), grid, dim3(512), 0, s, a);
  else if constexpr (D < 256) {
    if (p.row_waves == 1) hipLaunchKernelGGL((attend_kernel<TYPE, D, 2, 1>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((attend_kernel<TYPE, D, 2, 2>), grid, dim3(512), 0, s, a);
  }
  if (p.n_split > 1) {
    const int64_t rows = static_cast<int64_t>(a.b.n_seqs) * a.b.max_new * a.n_q_heads;
    // few rows of many parts by a workgroup each, many rows by a wave (63 parts of 32 rows: 4.7
    // us against 22; 8 of 8192: 18 against 9)
    if (p.n_split > 16) hipLaunchKernelGGL((join_kernel<TYPE, D, 4>), dim3(static_cast<unsigned>(rows)), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((join_kernel<TYPE, D, 1>), dim3(static_cast<unsigned>(cdiv(rows, 4))), dim3(256), 0, s, a);
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
  const Rows out_rows{out, n_tokens, 2 * width, 2 * ld_out};
  if (overlap(out_rows, Rows{q, n_tokens, 2 * width, 2 * ld_q}) || over_cache(out_rows, C)) return MOE_ERR_ARG;
  const Plan p = plan_of(C, n_q_heads, n_seqs, max_new, max_len);
  // threads of a launch
  if (cdiv(static_cast<int64_t>(n_seqs) * C->n_heads * p.n_split, 8) * 8 * p.row_blocks * (p.row_waves == 1 ? 256 : 512) > UINT32_MAX)
    return MOE_ERR_ARG;
  const int64_t all_rows = static_cast<int64_t>(n_seqs) * max_new * n_q_heads;
  float* part = static_cast<float*>(ws);
  const AttendArgs a{batch_of(C, table, max_pages, cache_len, n_seqs, new_off, n_tokens, max_new, status),
                     q, C->k, C->v, out, part, part + p.n_split * all_rows * C->head_dim, mask, ld_q, ld_out,
                     __builtin_fabsf(scale) * 1.44269504088896340736f, scale < 0.f ? 0x80008000u : 0u, n_q_heads,
                     n_q_heads / C->n_heads, mask_words, p.n_split, p.part_tiles, p.row_blocks, n_seqs * C->n_heads * p.n_split};
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (C->type == MOE_TYPE_BF16) launch<MOE_TYPE_BF16>(C->head_dim, p, s, a);
  else launch<MOE_TYPE_FP16>(C->head_dim, p, s, a);
  return launch_status(s);
}
