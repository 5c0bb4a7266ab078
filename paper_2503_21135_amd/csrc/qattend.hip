// qattend.hip -- moe_qcache_attention: softmax(scale q k) v of drafted tokens over a paged
// cache in 8 bits, each token seeing the cached tokens and the drafts its mask names.
//
// Rows, tiles and operands are laid out as in the 16-bit kernel (row r of a key/value head is
// draft r / G, query head g*G + r % G; S^T = K Q^T, O^T += V^T P^T; a lane owns one row), with
// steps of 64 keys, whose codes are as many bytes as 32 keys of 16 bits: a lane's 16 bytes are
// two operands' worth.  Keys: channels 64c + 16 grp + (0..15), taken by two products of 32
// channels each; the queries are read in the same order.  Values: slots 16 grp + (0..15).  Key
// tile kt takes keys 16*(r/4) + 4*kt + r%4 as its row r, which leaves lane group grp with the
// scores of keys 16 grp + (0..15), in order.
//
// Codes become bf16 or fp16 exactly.  With s_j and s'_j a key's and a value's scale, the second
// product's weight is w_j = p_j s'_j = 2^(score_j + log2 s'_j - m), m the row's maximum of these
// exponents, so that the largest weight of a row suits fp16 whatever the scales; the sum of
// p_j = w_j / s'_j stays fp32 (2^-64 <= s' <= 2^64).
#include <type_traits>

#include "attend.hpp"

namespace moe {
namespace cache {
namespace {

constexpr int kTile = 64;        // keys of a step; divides every page size
// A row's weights are 2^(exponent - maximum + kLift), with a maximum that may lag 2^kSlack
// behind: 2^15 at most, and normal fp16 numbers down to 2^-21 of the maximum.
constexpr float kSlack = 8.f, kLift = 7.f;

struct QArgs : AttendArgs {
  const float *ks, *vs;
};

// four codes of a word as two words of a 16-bit type: fp16 by the bits of 1024 + 128 + q, less
// 1152; bf16 through fp32, whose lower halves are zero for integers this small
template <int TYPE>
__device__ __forceinline__ void widen(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if constexpr (TYPE == MOE_TYPE_FP16) {
    const uint32_t b = w ^ 0x80808080u;
    const f16x2 off = {static_cast<_Float16>(-1152.f), static_cast<_Float16>(-1152.f)};
    lo = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, b, 0x04010400u)) + off);
    hi = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, b, 0x04030402u)) + off);
  } else {
    const float a = static_cast<float>(static_cast<int8_t>(w)), c = static_cast<float>(static_cast<int8_t>(w >> 8));
    const float d = static_cast<float>(static_cast<int8_t>(w >> 16)), e = static_cast<float>(static_cast<int8_t>(w >> 24));
    lo = __builtin_amdgcn_perm(__float_as_uint(c), __float_as_uint(a), 0x07060302u);
    hi = __builtin_amdgcn_perm(__float_as_uint(e), __float_as_uint(d), 0x07060302u);
  }
}
// the 8 codes of half `h` of a lane's 16 as an operand
template <int TYPE>
__device__ __forceinline__ u32x4 operand(const u32x4& w, int h) {
  u32x4 x;
  uint32_t a, b;
  widen<TYPE>(w[2 * h], a, b);
  x[0] = a;
  x[1] = b;
  widen<TYPE>(w[2 * h + 1], a, b);
  x[2] = a;
  x[3] = b;
  return x;
}

// Bits of the 16 drafts from d0 on (slots of cached tokens, seen by all, where negative) that token
// i (row t) sees, of its sequence's n.  Without branches: rows of a wave differ.
__device__ __forceinline__ uint32_t seen16(const QArgs& a, int64_t t, int i, int n, int d0) {
  const int d = max(d0, 0), below = min(max(-d0, 0), 16);
  uint32_t bits;
  if (a.mask) {     // the same for all
    const uint64_t* m = a.mask + t * a.mask_words;
    const int w = d >> 6, sh = d & 63;
    const uint64_t lo = m[min(w, a.mask_words - 1)], hi = m[min(w + 1, a.mask_words - 1)];
    bits = w < a.mask_words ? static_cast<uint32_t>(lo >> sh) : 0u;
    bits |= w + 1 < a.mask_words && sh ? static_cast<uint32_t>(hi << ((64 - sh) & 63)) : 0u;
  } else {
    bits = (1u << min(max(i - d + 1, 0), 16)) - 1;
  }
  bits &= (1u << min(max(n - d, 0), 16)) - 1;
  return (bits << below | ((1u << below) - 1)) & 0xFFFFu;
}

// log2 and reciprocal of a value's scale, of 2^-64 at least: a row of zeros that came with a scale of 0
// has its share of the sum, too.  (The logarithm of NaN, and of a negative scale, stays NaN.)
__device__ __forceinline__ float log_of(float s) { return __builtin_elementwise_maximum(__builtin_amdgcn_logf(s), -64.f); }
__device__ __forceinline__ float inverse_of(float s) { return fminf(__builtin_amdgcn_rcpf(s), 0x1p64f); }

// lane E's value of each 16 lanes, on all of them
template <int E>
__device__ __forceinline__ float from_lane(float v) { return dpp<0x150 + E>(v); }

// What a wave holds of its 16 RT rows.
template <int RT, int NV>
struct Rows16 {
  f32x4 o[RT][NV];
  float m[RT], ms[RT], l[RT];   // maximum, the same less the lift, sum
  int tok[RT];                  // this lane's row of each row tile: its draft

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int rt = 0; rt < RT; rt++) {
      m[rt] = ms[rt] = -INFINITY;
      l[rt] = 0.f;
#pragma unroll
      for (int v = 0; v < NV; v++) o[rt][v] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }

  // Scores of 64 keys into weights, in two steps for row tile rt: sc[kt][i] is this lane's row's
  // product with key 16 grp + 4 kt + i.  scales(kt) are those keys' scales times scale2, logs(kt) and
  // inverses(kt) log2 and reciprocal of their values' scales.
  // EDGE: slots that not everybody sees (drafts, or none at all) may be among them.
  template <bool EDGE, class S, class L>
  __device__ __forceinline__ void exponents(int rt, f32x4 (&sc)[4], S scales, L logs, uint32_t see) {
    float most = -INFINITY;
#pragma unroll
    for (int kt = 0; kt < 4; kt++) {
      const f32x4 k2 = scales(kt), lg = logs(kt);
#pragma unroll
      for (int i = 0; i < 4; i++) {
        float x = __fmaf_rn(sc[kt][i], k2[i], lg[i]);
        if constexpr (EDGE) x = see >> (4 * kt + i) & 1 ? x : -INFINITY;
        sc[kt][i] = x;
      }
      most = fmaxf(most, fmaxf(fmaxf(sc[kt][0], sc[kt][1]), fmaxf(sc[kt][2], sc[kt][3])));
    }
    // A row's maximum moves only when an exponent passes it by kSlack: until then no lane asks
    // the others for theirs.  (A row that has seen nothing has -infinity, which any passes.)
    if (__any(!(most <= ms[rt] + (kSlack + kLift)))) {
      const float all = rows_max(most);
      const bool moves = !(all <= ms[rt] + (kSlack + kLift));    // this row, whatever its neighbours do
      const float m2 = moves ? fmaxf(m[rt], all) : m[rt];
      const float ms2 = m2 == -INFINITY ? 0.f : m2 - kLift;
      const float f = m[rt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ms[rt] - ms2);
      l[rt] *= f;
#pragma unroll
      for (int v = 0; v < NV; v++)
#pragma unroll
        for (int i = 0; i < 4; i++) o[rt][v][i] *= f;
      m[rt] = m2;
      ms[rt] = m2 == -INFINITY ? -INFINITY : ms2;
    }
  }
  template <bool EDGE, bool REST, class V>
  __device__ __forceinline__ void weights(int rt, const f32x4 (&sc)[4], V inverses, uint32_t see, u32x4 (&pf)[2], u32x4 (&rest)[2]) {
    const float by = ms[rt] == -INFINITY ? 0.f : ms[rt];
#pragma unroll
    for (int kt = 0; kt < 4; kt++) {
      const f32x4 rv = inverses(kt);
      float p[4];
#pragma unroll
      for (int i = 0; i < 4; i++) {
        p[i] = __builtin_amdgcn_exp2f(sc[kt][i] - by);
        // the sum's terms stay fp32: of a row of values so small that the product is below fp16's
        // range, of zeros for one, it still takes the share of the softmax
        float r = __fmaf_rn(p[i], rv[i], l[rt]);
        if constexpr (EDGE) {
          p[i] = see >> (4 * kt + i) & 1 ? p[i] : 0.f;
          r = see >> (4 * kt + i) & 1 ? r : l[rt];
        }
        l[rt] = r;
      }
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        const uint32_t w = pack2<MOE_TYPE_FP16>(p[i], p[i + 1]);
        pf[kt >> 1][kt % 2 * 2 + i / 2] = w;
        if constexpr (REST) rest[kt >> 1][kt % 2 * 2 + i / 2] = pack2<MOE_TYPE_FP16>(p[i] - half_lo<MOE_TYPE_FP16>(w), p[i + 1] - half_hi<MOE_TYPE_FP16>(w));
      }
    }
  }
};

// Lane 16 grp + e's value of what belongs to keys 16 grp + (0..15), as keys 16 grp + 4 kt + (0..3) of
// each group's lanes.
__device__ __forceinline__ f32x4 from_lanes(float v, int kt) {
  if (kt == 0) return f32x4{from_lane<0>(v), from_lane<1>(v), from_lane<2>(v), from_lane<3>(v)};
  if (kt == 1) return f32x4{from_lane<4>(v), from_lane<5>(v), from_lane<6>(v), from_lane<7>(v)};
  if (kt == 2) return f32x4{from_lane<8>(v), from_lane<9>(v), from_lane<10>(v), from_lane<11>(v)};
  return f32x4{from_lane<12>(v), from_lane<13>(v), from_lane<14>(v), from_lane<15>(v)};
}

// Few rows, straight from memory: four waves on the same 16 RT rows, each with keys of its own.
// Many rows (RW > 1): RW waves on 16 RT rows each by KW groups of keys; a group's waves read its
// tiles once, side by side, and widen the codes once on their way into LDS (double-buffered,
// one barrier a tile).
// Few rows are bound by HBM: 64 single tokens by 32 query and 8 key heads of 128 over up to 4096, 415 MB,
// 83 us, 5.0 TB/s and up to 6.1 for longer contexts.  The next tile's
// keys load behind this one's products (else 94 us); a third wave a SIMD would spill (105).
// Many rows are bound by phases that hardly overlap: 4 trees of 64 over up to 32768 147 to 151 us (0.56 PFLOP/s;
// matrix instructions a third of a busy CU's cycles, vector ones half, LDS a third).  Tried for
// them: one row tile's products among the other's softmax 178 us, two workgroups a CU 179, the two waves of
// a SIMD half a tile apart 177, scales by lanes instead of LDS 170, s_setprio 172 (all against 161 then).
template <int TYPE, int D, int RT, int RW, int KW>
__global__ void __launch_bounds__(64 * RW * KW, RW * KW == 8 || (RW == 1 && D <= 128) ? 2 : 1) attend_kernel(QArgs a) {
  typedef elem_t<TYPE> E;
  constexpr int NV = D / 16, W = RW * KW;
  constexpr int TG = RW * kWave, NP = (4 * D + TG - 1) / TG;   // threads of a key group, 16-byte pieces of a tile's keys for each
  struct Tile {
    u32x4 k[kTile][D / 8];    // row 16 kt + col is the operand row of lane col in tile kt; pieces and rows are
    u32x4 v[D][kTile / 8];    // mixed so that 16 lanes' reads fall on all banks
    f32x4 k2[kTile / 4], lg[kTile / 4], rv[kTile / 4];
  };
  struct Sums { float x[W][16][D + 4]; };
  union Lds {
    Tile tile[2][KW];
    Sums sums;
  };
  constexpr bool kShared = RW > 1, kAhead = RT * D <= 128;
  // Weights are rounded to fp16, as outputs are or, in bf16, to less.  Few rows with fp16 outputs, which
  // wait for HBM, add the product with what the rounding left over; for many rows that would be half as much again
  // of the matrix work and of the weights' (4 trees of 64 over up to 32768: a call of 212 us instead of 157,
  // its error against 64 bits 2.1e-4, that of the output's rounding, instead of 2.9e-4).
  constexpr bool kRest = !kShared && TYPE == MOE_TYPE_FP16;
  __shared__ __attribute__((aligned(16))) char lds_bytes[kShared ? (KW > 1 ? sizeof(Lds) : sizeof(Tile) * 2) : sizeof(Sums)];
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

  // queries as operands of 32 channels, in the order that the keys' come in
  u32x4 qf[RT][D / 32];
  Rows16<RT, NV> st;
  st.clear();
#pragma unroll
  for (int rt = 0; rt < RT; rt++) {
    const int r = min(row0 + (wr * RT + rt) * 16 + col, rows - 1);   // a row past the last is its copy, not stored
    st.tok[rt] = r / a.group;
    const E* p = static_cast<const E*>(a.q) + (q.off + st.tok[rt]) * a.ld_q + (h * a.group + r % a.group) * D;
#pragma unroll
    for (int c = 0; c < D / 32; c++)
      qf[rt][c] = *reinterpret_cast<const u32x4*>(p + (kShared ? 32 * c + 8 * grp : 64 * (c / 2) + 16 * grp + 8 * (c % 2))) ^
                  u32x4{a.flip, a.flip, a.flip, a.flip};
  }
  auto see_of = [&](uint32_t (&see)[RT], int t) {
#pragma unroll
    for (int rt = 0; rt < RT; rt++) see[rt] = seen16(a, q.off + st.tok[rt], st.tok[rt], q.n, t * kTile + 16 * grp - q.len);
  };

  const int P = 1 << a.b.page_shift;
  // this wave's n-th tile, and the pages of 64 of them from the n-th on, one per lane
  constexpr int kStride = kShared ? KW : W;
  const int mine = kShared ? wk : wave;
  int pages = -1;
  auto look_up = [&](int n) {
    const int64_t tl = static_cast<int64_t>(t_first) + mine + static_cast<int64_t>(n + lane) * kStride;
    pages = tl < t_end ? page_of(a.b, s, static_cast<int>(tl) * kTile) : 0;
    if (pages < 0) report(a.b, MOE_ERR_SLOT);
  };
  // first slot of tile t in the head's memory, and the head's first
  auto head_at = [&](int page) { return (static_cast<int64_t>(page) * a.b.n_heads + h) * P; };
  const int t_full = min(t_end, q.len / kTile);    // tiles before it hold cached tokens alone

  if constexpr (!kShared) {
    const int krow = 16 * (col >> 2) + (col & 3);
    const uint32_t k_off = krow * D + 16 * grp, v_off = col * P + 16 * grp;
    auto load_k = [&](u32x4 (&kf)[4][D / 64], int page, int t) {
      const uint8_t* p = static_cast<const uint8_t*>(a.kc) + (head_at(max(page, 0)) + (t * kTile & (P - 1))) * D;
#pragma unroll
      for (int kt = 0; kt < 4; kt++)
#pragma unroll
        for (int c = 0; c < D / 64; c++) kf[kt][c] = *reinterpret_cast<const u32x4*>(p + (k_off + 4 * kt * D + 64 * c));
    };
    auto load_v = [&](u32x4 (&vf)[NV], float& ks, float& vs, int page, int t) {
      const int in_page = t * kTile & (P - 1);
      const int64_t head = head_at(max(page, 0));
      const uint8_t* p = static_cast<const uint8_t*>(a.vc) + head * D + in_page;
#pragma unroll
      for (int v = 0; v < NV; v++) vf[v] = *reinterpret_cast<const u32x4*>(p + 16 * v * P + v_off);
      ks = a.ks[head + in_page + lane];
      vs = a.vs[head + in_page + lane];
    };
    auto step = [&](auto edge_c, const u32x4 (&kf)[4][D / 64], const u32x4 (&vf)[NV], float ks, float vs, int t) {
      constexpr bool EDGE = decltype(edge_c)::value;
      uint32_t see[RT];
      if constexpr (EDGE) see_of(see, t);
      f32x4 sc[RT][4];
#pragma unroll
      for (int kt = 0; kt < 4; kt++) {
#pragma unroll
        for (int c = 0; c < D / 32; c++) {
          u32x4 codes = kf[kt][c / 2];
          asm("" : "+v"(codes));   // codes, not widened keys, are what waits for its turn in registers
          const u32x4 k = operand<TYPE>(codes, c % 2);
#pragma unroll
          for (int rt = 0; rt < RT; rt++) sc[rt][kt] = product<TYPE>(k, qf[rt][c], c ? sc[rt][kt] : f32x4{0.f, 0.f, 0.f, 0.f});
        }
      }
      u32x4 pf[RT][2], rest[RT][2];
      const float k2 = ks * a.scale2, lg = log_of(vs), rv = inverse_of(vs);
#pragma unroll
      for (int rt = 0; rt < RT; rt++) {
        st.template exponents<EDGE>(rt, sc[rt], [&](int kt) { return from_lanes(k2, kt); }, [&](int kt) { return from_lanes(lg, kt); }, see[rt]);
        st.template weights<EDGE, kRest>(rt, sc[rt], [&](int kt) { return from_lanes(rv, kt); }, see[rt], pf[rt], rest[rt]);
      }
#pragma unroll
      for (int v = 0; v < NV; v++)
#pragma unroll
        for (int e = 0; e < 2; e++) {
          const u32x4 w = operand<MOE_TYPE_FP16>(vf[v], e);
#pragma unroll
          for (int rt = 0; rt < RT; rt++) {
            st.o[rt][v] = product<MOE_TYPE_FP16>(w, pf[rt][e], st.o[rt][v]);
            if constexpr (kRest) st.o[rt][v] = product<MOE_TYPE_FP16>(w, rest[rt][e], st.o[rt][v]);
          }
        }
    };
    // the next tile's keys load behind this one's products; tiles with drafts in them, the
    // last ones, go one at a time
    int n = 0, t = t_first + wave;
    auto next_page = [&]() {
      if (++n % kWave == 0) look_up(n);
      return static_cast<int>(__builtin_amdgcn_readlane(pages, n % kWave));
    };
    look_up(0);
    int page = __builtin_amdgcn_readfirstlane(pages);
    u32x4 kf[4][D / 64], vf[NV];
    float ks, vs;
    if (t < t_full) {
      u32x4 kn[4][D / 64];
      load_k(kf, page, t);
      for (; t < t_full; t += W) {
        load_v(vf, ks, vs, page, t);
        const int next = next_page();
        if (kAhead && t + W < t_full) load_k(kn, next, t + W);
        if (page >= 0) step(std::false_type{}, kf, vf, ks, vs, t);
        if (!kAhead && t + W < t_full) load_k(kn, next, t + W);
#pragma unroll
        for (int kt = 0; kt < 4; kt++)
#pragma unroll
          for (int c = 0; c < D / 64; c++) kf[kt][c] = kn[kt][c];
        page = next;
      }
    }
#pragma unroll 1
    for (; t < t_end; t += W) {
      if (page >= 0) {
        load_k(kf, page, t);
        load_v(vf, ks, vs, page, t);
        step(std::true_type{}, kf, vf, ks, vs, t);
      }
      page = next_page();
    }
  } else {
    Lds& lds = *reinterpret_cast<Lds*>(lds_bytes);
    const int tid = threadIdx.x % TG;
    u32x4 kp[NP], vp[NP];
    float ks = 0.f, vs = 1.f;
    // loads of the group's r-th tile; whether it is there
    auto load = [&](int r) {
      if (r % kWave == 0) look_up(r);
      const int64_t t = static_cast<int64_t>(t_first) + wk + static_cast<int64_t>(r) * KW;
      const int page = __builtin_amdgcn_readlane(pages, r % kWave);
      if (t >= t_end || page < 0) return false;
      const int in_page = static_cast<int>(t) * kTile & (P - 1);
      const int64_t head = head_at(page);
      const uint8_t *kb = static_cast<const uint8_t*>(a.kc) + (head + in_page) * D, *vb = static_cast<const uint8_t*>(a.vc) + head * D + in_page;
#pragma unroll
      for (int i = 0; i < NP; i++) {
        const uint32_t x = tid + i * TG;
        if (x >= 4 * D) break;
        kp[i] = *reinterpret_cast<const u32x4*>(kb + x * 16);
        vp[i] = *reinterpret_cast<const u32x4*>(vb + ((x >> 2) * P + (x & 3) * 16));
      }
      if (tid < kTile) {
        ks = a.ks[head + in_page + tid];
        vs = a.vs[head + in_page + tid];
      }
      return true;
    };
    constexpr int kMix = D == 64 ? 7 : 15;
    auto mixed = [](int row) { return D == 64 ? row >> 1 & kMix : row & kMix; };
    bool there = load(0);
    const int stages = (t_end - t_first + KW - 1) / KW;
    auto stage = [&](auto edge_c, int r) {
      constexpr bool EDGE = decltype(edge_c)::value;
      Tile& tile = lds.tile[r & 1][wk];
      const bool now = there;
      if (now) {
#pragma unroll
        for (int i = 0; i < NP; i++) {
          const int x = tid + i * TG, key = x / (D / 16), row = 16 * (key >> 2 & 3) + 4 * (key >> 4) + (key & 3);
          const int c = x % (D / 16) * 2, vr = x >> 2, o = (x & 3) * 2;
          if (x >= 4 * D) break;
#pragma unroll
          for (int e = 0; e < 2; e++) {
            tile.k[row][(c + e) ^ mixed(row)] = operand<TYPE>(kp[i], e);
            tile.v[vr][(o + e) ^ (vr >> 1 & 7)] = operand<MOE_TYPE_FP16>(vp[i], e);
          }
        }
        if (tid < kTile) {
          tile.k2[tid / 4][tid % 4] = ks * a.scale2;
          tile.lg[tid / 4][tid % 4] = log_of(vs);
          tile.rv[tid / 4][tid % 4] = inverse_of(vs);
        }
      }
      __syncthreads();
      if (r + 1 < stages) there = load(r + 1);
      if (!now) return;
      const int t = t_first + wk + r * KW;
      uint32_t see[RT];
      if constexpr (EDGE) see_of(see, t);
      f32x4 sc[RT][4];
      u32x4 pf[RT][2];
#pragma unroll
      for (int kt = 0; kt < 4; kt++)
#pragma unroll
        for (int c = 0; c < D / 32; c++) {
          const u32x4 k = tile.k[16 * kt + col][(4 * c + grp) ^ mixed(col)];
#pragma unroll
          for (int rt = 0; rt < RT; rt++) sc[rt][kt] = product<TYPE>(k, qf[rt][c], c ? sc[rt][kt] : f32x4{0.f, 0.f, 0.f, 0.f});
        }
      if constexpr (D == 256) __builtin_amdgcn_sched_barrier(0);   // values read ahead would not fit
#pragma unroll
      for (int rt = 0; rt < RT; rt++)
        st.template exponents<EDGE>(rt, sc[rt], [&](int kt) { return tile.k2[4 * grp + kt]; }, [&](int kt) { return tile.lg[4 * grp + kt]; }, see[rt]);
#pragma unroll
      for (int rt = 0; rt < RT; rt++) st.template weights<EDGE, false>(rt, sc[rt], [&](int kt) { return tile.rv[4 * grp + kt]; }, see[rt], pf[rt], pf[rt]);
#pragma unroll
      for (int v = 0; v < NV; v++)
#pragma unroll
        for (int e = 0; e < 2; e++) {
          const u32x4 w = tile.v[16 * v + col][(2 * grp + e) ^ (col >> 1)];
#pragma unroll
          for (int rt = 0; rt < RT; rt++) st.o[rt][v] = product<MOE_TYPE_FP16>(w, pf[rt][e], st.o[rt][v]);
        }
    };
    const int full = max(0, t_full - t_first) / KW;   // stages whose tiles all hold cached tokens alone
    int r = 0;
    for (; r < full; r++) stage(std::false_type{}, r);
#pragma unroll 1
    for (; r < stages; r++) stage(std::true_type{}, r);
  }

  const int64_t all_rows = static_cast<int64_t>(a.b.n_seqs) * a.b.max_new * a.n_q_heads;
#pragma unroll
  for (int rt = 0; rt < RT; rt++) st.l[rt] = rows_sum(st.l[rt]);
  if constexpr (kShared && KW == 1) {    // a row's keys were all this wave's
#pragma unroll
    for (int rt = 0; rt < RT; rt++) {
      const int r = row0 + (wr * RT + rt) * 16 + col;
      if (r >= rows) continue;
      const int i_tok = r / a.group, head = h * a.group + r % a.group;
      if (a.n_split == 1) {
        const float inv = st.l[rt] == 0.f ? 0.f : 1.0f / st.l[rt];
        E* op = static_cast<E*>(a.out) + (q.off + i_tok) * a.ld_out + head * D + 4 * grp;
#pragma unroll
        for (int v = 0; v < NV; v++)
#pragma unroll
          for (int e = 0; e < 4; e++) op[16 * v + e] = static_cast<E>(st.o[rt][v][e] * inv);
      } else {
        const int64_t row = part * all_rows + (static_cast<int64_t>(s) * a.b.max_new + i_tok) * a.n_q_heads + head;
#pragma unroll
        for (int v = 0; v < NV; v++) *reinterpret_cast<f32x4*>(a.part + row * D + 16 * v + 4 * grp) = st.o[rt][v];
        if (grp == 0) {
          a.stat[2 * row] = st.m[rt];
          a.stat[2 * row + 1] = st.l[rt];
        }
      }
    }
    return;
  }
  // join the waves that shared the rows: common maximum, then the sums in wave order
  if constexpr (kShared) __syncthreads();    // the tiles' place is taken by the sums
  Sums& sums = *reinterpret_cast<Sums*>(lds_bytes);
  constexpr int KJ = kShared ? KW : W;       // waves of a row
#pragma unroll
  for (int rt = 0; rt < RT; rt++)
    if (grp == 0) {
      stats[wave][rt][col][0] = st.m[rt];
      stats[wave][rt][col][1] = st.l[rt];
    }
  __syncthreads();
#pragma unroll
  for (int rt = 0; rt < RT; rt++) {
    float top = -INFINITY;
    for (int w = 0; w < KJ; w++) top = fmaxf(top, stats[w * RW + wr][rt][col][0]);
    const float f = st.m[rt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st.m[rt] - top);
    if (rt) __syncthreads();
#pragma unroll
    for (int v = 0; v < NV; v++) {
      f32x4 x = st.o[rt][v];
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
      for (int w = 0; w < KJ; w++) hi = fmaxf(hi, stats[w * RW + w0][rt][rr][0]);
      f32x4 x = f32x4{0.f, 0.f, 0.f, 0.f};
      for (int w = 0; w < KJ; w++) {
        const float mw = stats[w * RW + w0][rt][rr][0];
        if (mw != -INFINITY) sum += stats[w * RW + w0][rt][rr][1] * __builtin_amdgcn_exp2f(mw - hi);
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

// How a batch is laid over workgroups.  Up to 16 rows (32 where the registers allow two tiles)
// per key head go straight from memory, more through LDS, whose tiles are shared by as many waves
// as there are row tiles.  Parts: as many as make the workgroups that are resident at once (four a
// CU of head_dim 64 straight from memory, two of 128, one otherwise), the nearest number to it,
// since a few too many run alone at the end (64 sequences by 8 heads of 128 over up to 4096: 84.0 us
// in 512 workgroups, 88.5 in 1024; 30 x 4 heads of 256 over 4000 62.3 in 240, 73.2 in 360; 6 x 8
// heads, 64 rows over 8000, 36.3 in 240, 50.8 in 288), and no shorter than two steps of every wave.
struct Plan {
  int row_waves;   // RW of the kernel
  int row_tiles;   // 16-row tiles of a wave
  int row_blocks;  // workgroups over the rows
  int n_split;     // parts of the keys
  int part_tiles;  // tiles of a part of the longest sequence
  int threads;     // of a workgroup
};

Plan plan_of(const moe_qcache_t* C, int n_q_heads, int n_seqs, int max_new, int max_len) {
  const int64_t rows = static_cast<int64_t>(max_new) * (n_q_heads / C->n_heads);
  const bool wide = C->head_dim == 256;
  Plan p;
  p.row_waves = rows <= (wide ? 16 : 32) ? 1 : rows <= (wide ? 64 : 128) ? 4 : 8;
  p.row_tiles = wide || (p.row_waves == 1 ? rows <= 16 : rows <= 64) ? 1 : 2;
  p.row_blocks = static_cast<int>(std::max<int64_t>(1, cdiv(rows, p.row_waves * p.row_tiles * 16)));
  const int key_waves = p.row_waves == 1 ? 4 : p.row_waves == 4 && !wide ? 2 : 1;
  p.threads = 64 * p.row_waves * key_waves;
  const int64_t wgs = std::max<int64_t>(1, static_cast<int64_t>(n_seqs) * C->n_heads * p.row_blocks);
  const int64_t tiles = std::max<int64_t>(1, cdiv(max_len, kTile)), slots = p.row_waves == 1 ? 65536 / C->head_dim : 256;
  const int64_t want = std::max<int64_t>(1, std::min<int64_t>({(slots + wgs / 2) / wgs, tiles / (2 * key_waves), kMaxSplit}));
  p.part_tiles = static_cast<int>(cdiv(tiles, want));
  p.n_split = static_cast<int>(cdiv(tiles, p.part_tiles));
  return p;
}

template <int TYPE, int D>
void launch(const Plan& p, hipStream_t s, const QArgs& a) {
  const dim3 grid(static_cast<unsigned>(cdiv(a.units, 8) * 8 * p.row_blocks));
  const dim3 block(p.threads);
  if constexpr (D == 256) {
    if (p.row_waves == 1) hipLaunchKernelGGL((attend_kernel<TYPE, D, 1, 1, 4>), grid, block, 0, s, a);
    else if (p.row_waves == 4) hipLaunchKernelGGL((attend_kernel<TYPE, D, 1, 4, 1>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((attend_kernel<TYPE, D, 1, 8, 1>), grid, block, 0, s, a);
  } else if (p.row_waves == 1) {
    if (p.row_tiles == 1) hipLaunchKernelGGL((attend_kernel<TYPE, D, 1, 1, 4>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((attend_kernel<TYPE, D, 2, 1, 4>), grid, block, 0, s, a);
  } else if (p.row_waves == 4) {
    if (p.row_tiles == 1) hipLaunchKernelGGL((attend_kernel<TYPE, D, 1, 4, 2>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((attend_kernel<TYPE, D, 2, 4, 2>), grid, block, 0, s, a);
  } else {
    hipLaunchKernelGGL((attend_kernel<TYPE, D, 2, 8, 1>), grid, block, 0, s, a);
  }
  if (p.n_split > 1) {
    const int64_t rows = static_cast<int64_t>(a.b.n_seqs) * a.b.max_new * a.n_q_heads;
    AttendArgs j = a;
    j.scale2 = 1.f;    // the parts' maxima are exponents already
    if (p.n_split > 16) hipLaunchKernelGGL((join_kernel<TYPE, D, kTile, 4>), dim3(static_cast<unsigned>(rows)), dim3(256), 0, s, j);
    else hipLaunchKernelGGL((join_kernel<TYPE, D, kTile, 1>), dim3(static_cast<unsigned>(cdiv(rows, 4))), dim3(256), 0, s, j);
  }
}

template <int TYPE>
void launch(int head_dim, const Plan& p, hipStream_t s, const QArgs& a) {
  if (head_dim == 64) launch<TYPE, 64>(p, s, a);
  else if (head_dim == 128) launch<TYPE, 128>(p, s, a);
  else launch<TYPE, 256>(p, s, a);
}

int check_sizes(const moe_qcache_t* C, int32_t n_q_heads, int32_t n_seqs, int32_t max_new, int32_t max_len) {
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

extern "C" int moe_qcache_attention_plan(const moe_qcache_t* C, int32_t n_q_heads, int32_t n_seqs,
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

extern "C" int moe_qcache_attention(const moe_qcache_t* C, const int32_t* table, int32_t max_pages,
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
  if (int st = moe_qcache_attention_plan(C, n_q_heads, n_seqs, max_new, max_len, nullptr, &need)) return st;
  if (need > 0 && (!ws || ws_bytes < need)) return MOE_ERR_WORKSPACE;
  if (need > 0 && !aligned16(ws)) return MOE_ERR_ALIGN;
  const Rows out_rows{out, n_tokens, 2 * width, 2 * ld_out};
  if (overlap(out_rows, Rows{q, n_tokens, 2 * width, 2 * ld_q}) || over_cache(out_rows, C)) return MOE_ERR_ARG;
  const Plan p = plan_of(C, n_q_heads, n_seqs, max_new, max_len);
  // threads of a launch
  if (cdiv(static_cast<int64_t>(n_seqs) * C->n_heads * p.n_split, 8) * 8 * p.row_blocks * p.threads > UINT32_MAX) return MOE_ERR_ARG;
  const int64_t all_rows = static_cast<int64_t>(n_seqs) * max_new * n_q_heads;
  float* part = static_cast<float*>(ws);
  QArgs a;
  static_cast<AttendArgs&>(a) = AttendArgs{
      batch_of(C, table, max_pages, cache_len, n_seqs, new_off, n_tokens, max_new, status), q, C->k, C->v, out, part,
      part + p.n_split * all_rows * C->head_dim, mask, ld_q, ld_out, __builtin_fabsf(scale) * 1.44269504088896340736f,
      scale < 0.f ? 0x80008000u : 0u, n_q_heads, n_q_heads / C->n_heads, mask_words, p.n_split, p.part_tiles, p.row_blocks,
      n_seqs * C->n_heads * p.n_split};
  a.ks = C->k_scale;
  a.vs = C->v_scale;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (C->type == MOE_TYPE_BF16) launch<MOE_TYPE_BF16>(C->head_dim, p, s, a);
  else launch<MOE_TYPE_FP16>(C->head_dim, p, s, a);
  return launch_status(s);
}
