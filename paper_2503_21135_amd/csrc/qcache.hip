// qcache.hip -- storing normed heads (moe_cache_append_norm), and the paged cache in 8 bits:
// moe_qcache_append, moe_qcache_read and moe_qcache_keep.
#include <algorithm>
#include <type_traits>

#include "cache.hpp"

namespace moe {
namespace cache {
namespace {

constexpr int kSlots = 64;      // slots of a workgroup, aligned
constexpr int kRowsKept = 32;   // rows a keep workgroup holds in registers at a time
constexpr float kLeast = 0x1p-64f, kMost = 0x1p64f;   // of a scale

struct StoreArgs {
  Batch b;
  const void *q, *k, *v;
  void *q_out, *kc, *vc;
  float *ks, *vs;
  const float *w_q, *w_k;
  const int32_t* positions;
  const float *cos, *sin;
  int64_t ld_q, ld_k, ld_v, ld_q_out;
  float eps;
  int group, rot_dim, max_pos, interleaved;
};

// 16 bytes at any address of a 16-bit type's row (global accesses need no alignment)
struct __attribute__((packed, aligned(2))) Piece { uint32_t w[4]; };

// over groups of N (4 to 32) side by side lanes, on all of them
template <int N>
__device__ __forceinline__ float group_sum(float v) {
  v += dpp<0xB1>(v);
  v += dpp<0x4E>(v);
  if constexpr (N >= 8) v += dpp<0x141>(v);
  if constexpr (N >= 16) v += dpp<0x140>(v);
  if constexpr (N >= 32) v += __shfl_xor(v, 16);
  return v;
}
template <int N>
__device__ __forceinline__ float group_max(float v) {
  v = fmaxf(v, dpp<0xB1>(v));
  v = fmaxf(v, dpp<0x4E>(v));
  if constexpr (N >= 8) v = fmaxf(v, dpp<0x141>(v));
  if constexpr (N >= 16) v = fmaxf(v, dpp<0x140>(v));
  if constexpr (N >= 32) v = fmaxf(v, __shfl_xor(v, 16));
  return v;
}

template <int TYPE>
__device__ __forceinline__ void unpack(const Piece& p, float* f) {
#pragma unroll
  for (int e = 0; e < 4; e++) {
    f[2 * e] = half_lo<TYPE>(p.w[e]);
    f[2 * e + 1] = half_hi<TYPE>(p.w[e]);
  }
}
template <int TYPE>
__device__ __forceinline__ Piece packed(const float* f) {
  Piece p;
#pragma unroll
  for (int e = 0; e < 4; e++) p.w[e] = pack2<TYPE>(f[2 * e], f[2 * e + 1]);
  return p;
}

// largest magnitude of N values, infinity where one is not finite
template <int N>
__device__ __forceinline__ float largest(const float* f) {
  float m = 0.f;
  bool bad = false;
#pragma unroll
  for (int e = 0; e < N; e++) {
    m = fmaxf(m, __builtin_fabsf(f[e]));
    bad = bad || !__builtin_isfinite(f[e]);
  }
  return bad ? INFINITY : m;
}
// a row's scale from its largest magnitude
__device__ __forceinline__ float scale_of(float m) {
  return m == INFINITY ? __builtin_nanf("") : fminf(fmaxf(m / 127.f, kLeast), kMost);
}
// Four codes, the first lowest.  A quotient by the scale's reciprocal is put right by its
// remainder: 16-bit values over their largest magnitude are often half-way between two codes.
// The sum with 1.5 * 2^23 leaves it rounded to an integer in the low bits; a row without a scale
// (NaN) gets the codes that fall out.
__device__ __forceinline__ uint32_t codes4(const float* f, float s, float inv) {
  uint32_t c[4];
#pragma unroll
  for (int e = 0; e < 4; e++) {
    const float y = f[e] * inv, x = __fmaf_rn(__fmaf_rn(-y, s, f[e]), inv, y);
    c[e] = __float_as_uint(__builtin_amdgcn_fmed3f(x, -127.f, 127.f) + 12582912.f);
  }
  const uint32_t lo = __builtin_amdgcn_perm(c[1], c[0], 0x0C0C0400u), hi = __builtin_amdgcn_perm(c[3], c[2], 0x04000C0Cu);
  return lo | hi;
}

// N floats of a row, at any address of one
template <int N>
__device__ __forceinline__ void load_floats(const float* p, float* f) {
  struct __attribute__((packed, aligned(4))) Four { float w[4]; };
#pragma unroll
  for (int i = 0; i < N / 4; i++) {
    const Four x = reinterpret_cast<const Four*>(p)[i];
#pragma unroll
    for (int e = 0; e < 4; e++) f[4 * i + e] = x.w[e];
  }
}

// One workgroup per 64 aligned slots of a sequence and key/value head g.  D / 16 lanes side by
// side take a head of one token, each a pair of its 8-channel chunks, the chunks that turn
// together, so that norm and largest magnitude are sums and maxima over a few lanes.  The
// tile's live tokens times its heads (the key's and the queries') are dealt out over the
// workgroup: a tree of few tokens has its heads side by side (one head of all 64 slots at a time: 32
// trees 15.9 us instead of 14, one token 4.7 instead of 3.4).  What the row's place alone tells is on
// its way before positions and pages are known, and the next head's row during this one's arithmetic.
// Prompts are bound by HBM: 8192 tokens of 32 query and 8 key heads of 128, 206 MB read and written,
// take 48.3 us in 16 bits (4.3 TB/s), 52.1 for 185 MB in 8, where a workgroup loads nothing while it quantizes.
// Trees of drafts (32 of 16 to 32 tokens: 14.2 to 14.7 us in 8 bits, 12.5 in 16) wait for a chain of dependent loads (lengths,
// pages and positions, rows), store their values a slot at a time, and leave half of the card idle: a tree
// has two tiles, the second mostly without a token, and tiles run fastest in the grid, so that workgroups with work
// all fall on every second XCD (with sequences fastest the call and its read took 17.8 us instead of 18.9).
// Values in workgroups of their own took the trees 15.8 us; six waves a SIMD spill.
template <int TYPE, int D, bool Q8>
__global__ void __launch_bounds__(4 * D) store_kernel(StoreArgs a) {
  typedef elem_t<TYPE> E;
  constexpr int kItems = D / 16;        // pairs of 8-channel chunks of a head
  constexpr int kPiece = Q8 ? 16 : 8;   // slots of a value channel's 16 bytes
  constexpr int kDirect = 16;           // up to so many new tokens of a tile, values go to their places without LDS
  typedef std::conditional_t<Q8, uint16_t, uint32_t> Two;   // two slots of a channel
  __shared__ int64_t pages[kSlots / 32];            // first slot of each 32 in the head of its page, or -1
  __shared__ int where[kSlots];                     // position of each slot's token, or -1: no token, or one to skip
  __shared__ Two turned[D][kSlots / 2 + 2];
  // w_k and w_q: in registers instead a call of 8192 tokens by 32 and 8 heads of 128 takes 50.3 us, not 49.1, and
  // one of 8 x 300 to 600 tokens by 16 and 4 heads of 256 52.3, not 49.6
  __shared__ __attribute__((aligned(16))) float norms[2][D];
  const int s = blockIdx.y, g = blockIdx.z, tid = threadIdx.x;
  bool ok;
  const Seq q = sequence(a.b, s, ok);
  if (!ok && tid == 0) report(a.b, MOE_ERR_SLOT);
  const int P = 1 << a.b.page_shift;
  const int64_t first = q.len / kSlots * kSlots + static_cast<int64_t>(blockIdx.x) * kSlots;
  const int end = q.len + q.n;
  if (first >= end) return;
  const int slot0 = static_cast<int>(first);
  const int64_t t0 = static_cast<int64_t>(q.off) - q.len + slot0;   // token of the tile's first slot
  auto live = [&](int o) { return slot0 + o >= q.len && slot0 + o < end; };

  // values: each thread two slots by 8 channels
  const int vc8 = tid % (D / 8) * 8, pair = tid / (D / 8);
  Piece val[2] = {};
#pragma unroll
  for (int e = 0; e < 2; e++)
    if (live(2 * pair + e))
      val[e] = *reinterpret_cast<const Piece*>(static_cast<const E*>(a.v) + (t0 + 2 * pair + e) * a.ld_v + g * D + vc8);
  // keys and queries
  const int half = a.rot_dim / 2, j = tid % kItems;
  const bool turn = a.cos && 16 * j < a.rot_dim;
  const bool split = turn && !a.interleaved;    // chunks half a rotation apart
  const int c0 = split ? 8 * j : 16 * j, c1 = split ? half + 8 * j : 16 * j + 8;
  const int o_first = max(q.len - slot0, 0), n_live = min(end - slot0, kSlots) - o_first;
  const int items = n_live * (a.q ? a.group + 1 : 1);   // item i: head i / n_live (0 the key's) of live token i % n_live
  Piece x = {}, y = {};
  auto load_item = [&](int i) {
    const int head = i / n_live;
    const int64_t t = t0 + o_first + (i - head * n_live);
    const E* p = head == 0 ? static_cast<const E*>(a.k) + t * a.ld_k + g * D
                           : static_cast<const E*>(a.q) + t * a.ld_q + (static_cast<int64_t>(g) * a.group + head - 1) * D;
    x = *reinterpret_cast<const Piece*>(p + c0);
    y = *reinterpret_cast<const Piece*>(p + c1);
  };
  int item = tid / kItems;
  if (item < items) load_item(item);
  if (const float* from = tid < D ? a.w_k : tid < 2 * D ? a.w_q : nullptr) norms[tid / D][tid % D] = from[tid % D];

  if (tid < kSlots) {
    const int slot = slot0 + tid;
    const int pos = !live(tid) ? -1 : (a.positions ? a.positions[t0 + tid] : slot);
    const bool bad = live(tid) && a.cos && (pos < 0 || pos >= a.max_pos);
    where[tid] = live(tid) && !bad ? (a.cos ? pos : 0) : -1;
    bool lost = false;
    if (tid % 32 == 0) {
      const int page = slot < end && slot + 32 > q.len ? page_of(a.b, s, slot) : 0;
      lost = page < 0;
      pages[tid / 32] = lost ? -1 : (static_cast<int64_t>(page) * a.b.n_heads + g) * P + (slot & (P - 1));
    }
    if (bad || lost) report(a.b, MOE_ERR_SLOT);
  }
  __syncthreads();

  float cs[8], sn[8];
  int o_of = -1;        // the token that they are of
  for (; item < items; item += kSlots) {
    const int head = item / n_live, o = o_first + (item - head * n_live), pos = where[o];
    float f[16];
    unpack<TYPE>(x, f);
    unpack<TYPE>(y, f + 8);
    if (turn && pos >= 0 && o != o_of) {   // before the next row, which is not waited for then
      const int64_t at = static_cast<int64_t>(pos) * half + 8 * j;
      load_floats<8>(a.cos + at, cs);
      load_floats<8>(a.sin + at, sn);
      o_of = o;
    }
    if (item + kSlots < items) load_item(item + kSlots);
    if (pos < 0) continue;
    if (head ? a.w_q : a.w_k) {
      float w[16];
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(&norms[head > 0][(e < 8 ? c0 : c1) + e % 8]);
#pragma unroll
        for (int i = 0; i < 4; i++) w[e + i] = x[i];
      }
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < 16; e++) ss = __fmaf_rn(f[e], f[e], ss);
      const float r = __builtin_amdgcn_rsqf(group_sum<kItems>(ss) * (1.0f / D) + a.eps);
#pragma unroll
      for (int e = 0; e < 16; e++) f[e] = f[e] * r * w[e];
    }
    if (turn) {
      auto rotated = [&](float& u, float& v, int e) {
        const float s = __fmaf_rn(u, cs[e], -(v * sn[e])), t = __fmaf_rn(u, sn[e], v * cs[e]);
        u = s;
        v = t;
      };
      if (a.interleaved) {
#pragma unroll
        for (int e = 0; e < 8; e++) rotated(f[2 * e], f[2 * e + 1], e);
      } else {
#pragma unroll
        for (int e = 0; e < 8; e++) rotated(f[e], f[8 + e], e);
      }
    }
    if (head) {
      E* op = static_cast<E*>(a.q_out) + (t0 + o) * a.ld_q_out + (static_cast<int64_t>(g) * a.group + head - 1) * D;
      *reinterpret_cast<Piece*>(op + c0) = packed<TYPE>(f);
      *reinterpret_cast<Piece*>(op + c1) = packed<TYPE>(f + 8);
      continue;
    }
    const int64_t page = pages[o / 32], slot = page + o % 32;
    if (page < 0) continue;
    if constexpr (Q8) {
      const float s = scale_of(group_max<kItems>(largest<16>(f))), inv = 1.0f / s;
      if (j == 0) a.ks[slot] = s;
      uint8_t* out = static_cast<uint8_t*>(a.kc) + slot * D;
      *reinterpret_cast<u32x2*>(out + c0) = u32x2{codes4(f, s, inv), codes4(f + 4, s, inv)};
      *reinterpret_cast<u32x2*>(out + c1) = u32x2{codes4(f + 8, s, inv), codes4(f + 12, s, inv)};
    } else {
      E* out = static_cast<E*>(a.kc) + slot * D;
      *reinterpret_cast<Piece*>(out + c0) = packed<TYPE>(f);
      *reinterpret_cast<Piece*>(out + c1) = packed<TYPE>(f + 8);
    }
  }

  // the thread's values as they are stored, [slot][two channels or four] to a word
  uint32_t kept[2][Q8 ? 2 : 4];
#pragma unroll
  for (int e = 0; e < 2; e++) {
    if constexpr (Q8) {
      float f[8];
      unpack<TYPE>(val[e], f);
      const float s = scale_of(group_max<D / 8>(largest<8>(f))), inv = 1.0f / s;
      kept[e][0] = codes4(f, s, inv);
      kept[e][1] = codes4(f + 4, s, inv);
      const int o = 2 * pair + e;
      if (vc8 == 0 && where[o] >= 0 && pages[o / 32] >= 0) a.vs[pages[o / 32] + o % 32] = s;
    } else {
#pragma unroll
      for (int i = 0; i < 4; i++) kept[e][i] = val[e].w[i];
    }
  }
  typedef std::conditional_t<Q8, uint8_t, uint16_t> One;
  constexpr int kBits = 8 * sizeof(One), kPer = 32 / kBits;
  auto value = [&](int e, int i) { return static_cast<One>(kept[e][i / kPer] >> kBits * (i % kPer)); };
  // head's values of the page of slot o's 32, at that slot
  auto home = [&](int o, int c) {
    const int64_t page = pages[o / 32];
    const int64_t in_page = page & (P - 1);
    return static_cast<One*>(a.vc) + (page - in_page) * D + static_cast<int64_t>(c) * P + in_page + o % 32;
  };
  if (min(end, slot0 + kSlots) - max(q.len, slot0) <= kDirect) {
#pragma unroll
    for (int e = 0; e < 2; e++) {
      const int o = 2 * pair + e;
      if (where[o] < 0 || pages[o / 32] < 0) continue;
      One* out = home(o, vc8);
#pragma unroll
      for (int i = 0; i < 8; i++) out[static_cast<int64_t>(i) * P] = value(e, i);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; i++)
    turned[vc8 + i][pair] = static_cast<Two>(value(0, i) | static_cast<uint32_t>(value(1, i)) << kBits);
  __syncthreads();
  for (int i = tid; i < D * (kSlots / kPiece); i += 4 * D) {
    const int o = i % (kSlots / kPiece) * kPiece, c = i / (kSlots / kPiece);
    if (slot0 + o + kPiece <= q.len || slot0 + o >= end || pages[o / 32] < 0) continue;
    One* out = home(o, c);
    bool all = true;
#pragma unroll
    for (int e = 0; e < kPiece; e++) all = all && where[o + e] >= 0;
    const One* from = reinterpret_cast<const One*>(&turned[c][0]) + o;
    if (all) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; e++) w[e] = reinterpret_cast<const uint32_t*>(from)[e];
      *reinterpret_cast<u32x4*>(out) = w;
    } else {
#pragma unroll
      for (int w = 0; w < kPiece; w += kPer) {    // words whose slots are all new, or their slots
        bool word = true;
#pragma unroll
        for (int e = 0; e < kPer; e++) word = word && where[o + w + e] >= 0;
        if (word) *reinterpret_cast<uint32_t*>(out + w) = *reinterpret_cast<const uint32_t*>(from + w);
#pragma unroll
        for (int e = 0; e < kPer; e++)
          if (!word && where[o + w + e] >= 0) out[w + e] = from[w + e];
      }
    }
  }
}

struct ReadArgs {
  Batch b;             // len: the first slot, off: the rows
  const void *kc, *vc;
  const float *ks, *vs;
  void *k_out, *v_out;
  int64_t ld_k, ld_v;
};

template <int TYPE>
__device__ __forceinline__ uint32_t two(uint32_t codes, int i, float s) {   // codes i and i + 1 of a word times s
  const float a = static_cast<float>(static_cast<int8_t>(codes >> 8 * i)), b = static_cast<float>(static_cast<int8_t>(codes >> (8 * i + 8)));
  return pack2<TYPE>(a * s, b * s);
}

// One workgroup per 64 aligned slots of a sequence and head; values turn over through LDS, so that
// both sides of the copy move 16 bytes a lane.  Bound by HBM (8192 rows of 8 heads of 128, 51 MB,
// 11.3 us, 4.5 TB/s) or, for few rows, by the latency of its loads (the rows of 32 trees 5.1 us).
template <int TYPE, int D>
__global__ void __launch_bounds__(256) read_kernel(ReadArgs a) {
  typedef elem_t<TYPE> E;
  __shared__ uint32_t codes[D][kSlots / 4 + 1];
  __shared__ float scale[kSlots];
  const int s = blockIdx.y, g = blockIdx.z, tid = threadIdx.x;
  bool ok;
  const Seq q = sequence(a.b, s, ok);
  if (!ok && tid == 0) report(a.b, MOE_ERR_SLOT);
  const int P = 1 << a.b.page_shift;
  const int64_t first = q.len / kSlots * kSlots + static_cast<int64_t>(blockIdx.x) * kSlots;
  const int end = q.len + q.n;
  if (first >= end) return;
  const int slot0 = static_cast<int>(first);
  const int page = page_of(a.b, s, slot0);
  if (page < 0) {
    if (tid == 0) report(a.b, MOE_ERR_SLOT);
    return;
  }
  const int64_t head = (static_cast<int64_t>(page) * a.b.n_heads + g) * P;
  const int in_page = slot0 & (P - 1);
  const int64_t t0 = static_cast<int64_t>(q.off) - q.len + slot0;
  auto live = [&](int o) { return slot0 + o >= q.len && slot0 + o < end; };
  if (a.k_out)
    for (int i = tid; i < kSlots * (D / 16); i += 256) {
      const int o = i / (D / 16), c = i % (D / 16) * 16;
      if (!live(o)) continue;
      const float sc = a.ks[head + in_page + o];
      const u32x4 w = *reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(a.kc) + (head + in_page + o) * D + c);
      E* out = static_cast<E*>(a.k_out) + (t0 + o) * a.ld_k + g * D + c;
#pragma unroll
      for (int p = 0; p < 2; p++) {
        Piece x;
#pragma unroll
        for (int e = 0; e < 4; e++) x.w[e] = two<TYPE>(w[2 * p + e / 2], e % 2 * 2, sc);
        *reinterpret_cast<Piece*>(out + 8 * p) = x;
      }
    }
  if (!a.v_out) return;
  if (tid < kSlots) scale[tid] = live(tid) ? a.vs[head + in_page + tid] : 0.f;
  for (int i = tid; i < D * 4; i += 256) {
    const int c = i / 4, o = i % 4 * 16;
    if (slot0 + o + 16 <= q.len || slot0 + o >= end) continue;
    const u32x4 w = *reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(a.vc) + head * D + static_cast<int64_t>(c) * P + in_page + o);
#pragma unroll
    for (int e = 0; e < 4; e++) codes[c][o / 4 + e] = w[e];
  }
  __syncthreads();
  for (int i = tid; i < kSlots * (D / 8); i += 256) {
    const int o = i / (D / 8), c = i % (D / 8) * 8;
    if (!live(o)) continue;
    const float sc = scale[o];
    Piece x;
#pragma unroll
    for (int e = 0; e < 4; e++) {
      const int8_t lo = static_cast<int8_t>(codes[c + 2 * e][o / 4] >> 8 * (o % 4)), hi = static_cast<int8_t>(codes[c + 2 * e + 1][o / 4] >> 8 * (o % 4));
      x.w[e] = pack2<TYPE>(static_cast<float>(lo) * sc, static_cast<float>(hi) * sc);
    }
    *reinterpret_cast<Piece*>(static_cast<E*>(a.v_out) + (t0 + o) * a.ld_v + g * D + c) = x;
  }
}

struct KeepArgs {
  Batch b;
  void *kc, *vc;
  float *ks, *vs;
  const int32_t *keep, *n_keep;
  int32_t* len_out;
  int max_keep;
};

// One workgroup per sequence and head.  Rows go 32 at a time through registers, all read
// before any is written; indices ascend, so no later row's source is written before
// it is read.  Rows that stay where they are are left alone.  Cache lines bound it: a moved row's
// values touch head_dim of them for a byte each (256 trees by 8 heads of 128 12.7 us; one tree, a
// chain of loads, 4.1).
template <int D>
__global__ void __launch_bounds__(256) keep_kernel(KeepArgs a) {
  constexpr int kVec = (kRowsKept * (D / 16) + 255) / 256;   // 16-byte pieces of key rows per thread
  constexpr int kVals = kRowsKept * D / 256;                 // values per thread
  __shared__ int64_t from[kRowsKept], to[kRowsKept];         // head starts in slots, from < 0: nothing to move
  __shared__ int from_slot[kRowsKept], to_slot[kRowsKept];
  const int s = blockIdx.x, h = blockIdx.y, tid = threadIdx.x;
  bool ok;
  const Seq q = sequence(a.b, s, ok);
  const int n = a.n_keep[s];
  const int32_t* list = a.keep + static_cast<int64_t>(s) * a.max_keep;
  ok = ok && n >= 0 && n <= a.max_keep;
  bool bad = false;
  for (int j = tid; ok && j < n; j += 256) bad = bad || list[j] < 0 || list[j] >= q.n || (j > 0 && list[j] <= list[j - 1]);
  ok = !__syncthreads_or(bad) && ok;
  if (tid == 0 && h == 0) {
    if (!ok) report(a.b, MOE_ERR_SLOT);
    if (a.len_out) a.len_out[s] = a.b.len[s] + (ok ? n : 0);
  }
  if (!ok) return;
  const int P = 1 << a.b.page_shift;
  uint8_t *kc = static_cast<uint8_t*>(a.kc), *vc = static_cast<uint8_t*>(a.vc);
  for (int j0 = 0; j0 < n; j0 += kRowsKept) {
    __syncthreads();
    if (tid < kRowsKept) {
      const int j = j0 + tid;
      int64_t f = -1;
      if (j < n && list[j] != j) {
        const int fs = q.len + list[j], ts = q.len + j;
        const int pf = page_of(a.b, s, fs), pt = page_of(a.b, s, ts);
        if (pf < 0 || pt < 0) {
          report(a.b, MOE_ERR_SLOT);
        } else {
          f = (static_cast<int64_t>(pf) * a.b.n_heads + h) * P;
          to[tid] = (static_cast<int64_t>(pt) * a.b.n_heads + h) * P;
          from_slot[tid] = fs & (P - 1);
          to_slot[tid] = ts & (P - 1);
        }
      }
      from[tid] = f;
    }
    __syncthreads();
    u32x4 key[kVec];
    uint8_t val[kVals];
    float scale = 0.f;
    const float* scales = tid < kRowsKept ? a.ks : a.vs;   // threads 0..31 and 32..63
    const int sr = tid % kRowsKept;
    if (tid < 2 * kRowsKept && from[sr] >= 0) scale = scales[from[sr] + from_slot[sr]];
#pragma unroll
    for (int i = 0; i < kVec; i++) {
      const int x = tid + i * 256, row = x / (D / 16), c = x % (D / 16) * 16;
      if (row < kRowsKept && from[row] >= 0) key[i] = *reinterpret_cast<const u32x4*>(kc + (from[row] + from_slot[row]) * D + c);
    }
#pragma unroll
    for (int i = 0; i < kVals; i++) {
      const int row = tid % 8 + i % (kRowsKept / 8) * 8, c = tid / 8 + i / (kRowsKept / 8) * 32;
      if (from[row] >= 0) val[i] = vc[from[row] * D + static_cast<int64_t>(c) * P + from_slot[row]];
    }
    __syncthreads();
    if (tid < 2 * kRowsKept && from[sr] >= 0) (tid < kRowsKept ? a.ks : a.vs)[to[sr] + to_slot[sr]] = scale;
#pragma unroll
    for (int i = 0; i < kVec; i++) {
      const int x = tid + i * 256, row = x / (D / 16), c = x % (D / 16) * 16;
      if (row < kRowsKept && from[row] >= 0) *reinterpret_cast<u32x4*>(kc + (to[row] + to_slot[row]) * D + c) = key[i];
    }
#pragma unroll
    for (int i = 0; i < kVals; i++) {
      const int row = tid % 8 + i % (kRowsKept / 8) * 8, c = tid / 8 + i / (kRowsKept / 8) * 32;
      if (from[row] >= 0) vc[to[row] * D + static_cast<int64_t>(c) * P + to_slot[row]] = val[i];
    }
  }
}

template <int TYPE, bool Q8>
void launch_store(int head_dim, dim3 grid, hipStream_t s, const StoreArgs& a) {
  if (head_dim == 64) hipLaunchKernelGGL((store_kernel<TYPE, 64, Q8>), grid, dim3(4 * 64), 0, s, a);
  else if (head_dim == 128) hipLaunchKernelGGL((store_kernel<TYPE, 128, Q8>), grid, dim3(4 * 128), 0, s, a);
  else hipLaunchKernelGGL((store_kernel<TYPE, 256, Q8>), grid, dim3(4 * 256), 0, s, a);
}

// tiles of 64 aligned slots that n slots in a row can touch
unsigned tiles_of(int n) { return static_cast<unsigned>((static_cast<int64_t>(n) + kSlots - 2) / kSlots + 1); }

// the two appends, of a cache in 16 or 8 bits
template <class CACHE>
int store(const CACHE* C, const int32_t* table, int32_t max_pages, const int32_t* cache_len, int32_t n_seqs,
          const int32_t* new_off, int32_t n_tokens, int32_t max_new, const void* q, int64_t ld_q, int32_t n_q_heads,
          const void* k, int64_t ld_k, const void* v, int64_t ld_v, const float* w_q, const float* w_k, float eps,
          const int32_t* positions, const float* cos, const float* sin, int32_t rot_dim, int32_t max_pos,
          int32_t interleaved, void* q_out, int64_t ld_q_out, int32_t* status, void* stream) {
  if (int st = check_cache(C)) return st;
  if (n_seqs < 0 || n_seqs > 65535 || n_tokens < 0 || max_new < 0 || !(eps >= 0.f)) return MOE_ERR_ARG;
  if (n_seqs == 0 || n_tokens == 0 || max_new == 0) return MOE_OK;
  if (int st = check_batch(C, table, max_pages, cache_len, new_off)) return st;
  const int D = C->head_dim;
  max_new = std::min(max_new, n_tokens);
  if (!k || !v || ld_k < static_cast<int64_t>(C->n_heads) * D || ld_v < static_cast<int64_t>(C->n_heads) * D)
    return MOE_ERR_ARG;
  if (!q != !q_out) return MOE_ERR_ARG;
  if (q && (n_q_heads < 1 || n_q_heads % C->n_heads || ld_q < static_cast<int64_t>(n_q_heads) * D || ld_q_out < static_cast<int64_t>(n_q_heads) * D ||
            (q == q_out && ld_q != ld_q_out)))
    return MOE_ERR_ARG;
  if (!cos != !sin || (cos && (rot_dim < 16 || rot_dim % 16 || rot_dim > D || max_pos < 1))) return MOE_ERR_ARG;
  if (!aligned_to(q, 2) || !aligned_to(k, 2) || !aligned_to(v, 2) || !aligned_to(q_out, 2) || !aligned_to(cos, 4) ||
      !aligned_to(sin, 4) || !aligned_to(positions, 4) || !aligned_to(w_q, 4) || !aligned_to(w_k, 4))
    return MOE_ERR_ALIGN;
  if (q) {
    const int64_t wide = 2 * static_cast<int64_t>(n_q_heads) * D, slim = 2 * static_cast<int64_t>(C->n_heads) * D;
    const Rows out{q_out, n_tokens, wide, 2 * ld_q_out};
    if ((q != q_out && overlap(out, Rows{q, n_tokens, wide, 2 * ld_q})) || overlap(out, Rows{k, n_tokens, slim, 2 * ld_k}) ||
        overlap(out, Rows{v, n_tokens, slim, 2 * ld_v}) || over_cache(out, C))
      return MOE_ERR_ARG;
  }
  StoreArgs a{batch_of(C, table, max_pages, cache_len, n_seqs, new_off, n_tokens, max_new, status),
              q, k, v, q_out, C->k, C->v, nullptr, nullptr, w_q, w_k, positions, cos, sin, ld_q, ld_k, ld_v, ld_q_out,
              eps, n_q_heads / C->n_heads, rot_dim, max_pos, interleaved};
  const dim3 grid(tiles_of(max_new), n_seqs, C->n_heads);
  hipStream_t s = static_cast<hipStream_t>(stream);
  constexpr bool Q8 = std::is_same_v<CACHE, moe_qcache_t>;
  if constexpr (Q8) {
    a.ks = C->k_scale;
    a.vs = C->v_scale;
  }
  if (C->type == MOE_TYPE_BF16) launch_store<MOE_TYPE_BF16, Q8>(D, grid, s, a);
  else launch_store<MOE_TYPE_FP16, Q8>(D, grid, s, a);
  return launch_status(s);
}

}  // namespace
}  // namespace cache
}  // namespace moe

extern "C" int moe_cache_append_norm(const moe_cache_t* C, const int32_t* table, int32_t max_pages,
                                     const int32_t* cache_len, int32_t n_seqs, const int32_t* new_off,
                                     int32_t n_tokens, int32_t max_new, const void* q, int64_t ld_q,
                                     int32_t n_q_heads, const void* k, int64_t ld_k, const void* v,
                                     int64_t ld_v, const float* w_q, const float* w_k, float eps,
                                     const int32_t* positions, const float* cos, const float* sin,
                                     int32_t rot_dim, int32_t max_pos, int32_t interleaved,
                                     void* q_out, int64_t ld_q_out, int32_t* status, void* stream) {
  return moe::cache::store(C, table, max_pages, cache_len, n_seqs, new_off, n_tokens, max_new, q, ld_q, n_q_heads, k, ld_k,
                           v, ld_v, w_q, w_k, eps, positions, cos, sin, rot_dim, max_pos, interleaved, q_out, ld_q_out, status, stream);
}

extern "C" int moe_qcache_append(const moe_qcache_t* C, const int32_t* table, int32_t max_pages,
                                 const int32_t* cache_len, int32_t n_seqs, const int32_t* new_off,
                                 int32_t n_tokens, int32_t max_new, const void* q, int64_t ld_q,
                                 int32_t n_q_heads, const void* k, int64_t ld_k, const void* v,
                                 int64_t ld_v, const float* w_q, const float* w_k, float eps,
                                 const int32_t* positions, const float* cos, const float* sin,
                                 int32_t rot_dim, int32_t max_pos, int32_t interleaved,
                                 void* q_out, int64_t ld_q_out, int32_t* status, void* stream) {
  return moe::cache::store(C, table, max_pages, cache_len, n_seqs, new_off, n_tokens, max_new, q, ld_q, n_q_heads, k, ld_k,
                           v, ld_v, w_q, w_k, eps, positions, cos, sin, rot_dim, max_pos, interleaved, q_out, ld_q_out, status, stream);
}

extern "C" int moe_qcache_read(const moe_qcache_t* C, const int32_t* table, int32_t max_pages,
                               const int32_t* first, int32_t n_seqs, const int32_t* row_off, int32_t n_rows,
                               int32_t max_rows, void* k_out, int64_t ld_k_out, void* v_out, int64_t ld_v_out,
                               int32_t* status, void* stream) {
  using namespace moe;
  using namespace moe::cache;
  if (int st = check_cache(C)) return st;
  if (n_seqs < 0 || n_seqs > 65535 || n_rows < 0 || max_rows < 0) return MOE_ERR_ARG;
  if (n_seqs == 0 || n_rows == 0 || max_rows == 0) return MOE_OK;
  if (int st = check_batch(C, table, max_pages, first, row_off)) return st;
  const int64_t width = static_cast<int64_t>(C->n_heads) * C->head_dim;
  if ((!k_out && !v_out) || (k_out && ld_k_out < width) || (v_out && ld_v_out < width)) return MOE_ERR_ARG;
  if (!aligned_to(k_out, 2) || !aligned_to(v_out, 2)) return MOE_ERR_ALIGN;
  const Rows k{k_out, n_rows, 2 * width, 2 * ld_k_out}, v{v_out, n_rows, 2 * width, 2 * ld_v_out};
  if ((k_out && v_out && overlap(k, v)) || (k_out && over_cache(k, C)) || (v_out && over_cache(v, C))) return MOE_ERR_ARG;
  const ReadArgs a{batch_of(C, table, max_pages, first, n_seqs, row_off, n_rows, max_rows, status),
                   C->k, C->v, C->k_scale, C->v_scale, k_out, v_out, ld_k_out, ld_v_out};
  const dim3 grid(tiles_of(std::min(max_rows, n_rows)), n_seqs, C->n_heads), block(256);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool bf = C->type == MOE_TYPE_BF16;
  if (C->head_dim == 64) {
    if (bf) hipLaunchKernelGGL((read_kernel<MOE_TYPE_BF16, 64>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((read_kernel<MOE_TYPE_FP16, 64>), grid, block, 0, s, a);
  } else if (C->head_dim == 128) {
    if (bf) hipLaunchKernelGGL((read_kernel<MOE_TYPE_BF16, 128>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((read_kernel<MOE_TYPE_FP16, 128>), grid, block, 0, s, a);
  } else {
    if (bf) hipLaunchKernelGGL((read_kernel<MOE_TYPE_BF16, 256>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((read_kernel<MOE_TYPE_FP16, 256>), grid, block, 0, s, a);
  }
  return launch_status(s);
}

extern "C" int moe_qcache_keep(const moe_qcache_t* C, const int32_t* table, int32_t max_pages,
                               const int32_t* cache_len, int32_t n_seqs, const int32_t* new_off,
                               const int32_t* keep, int32_t max_keep, const int32_t* n_keep,
                               int32_t* len_out, int32_t* status, void* stream) {
  using namespace moe;
  using namespace moe::cache;
  if (int st = check_cache(C)) return st;
  if (n_seqs < 0 || n_seqs > 65535 || max_keep < 0) return MOE_ERR_ARG;
  if (n_seqs == 0) return MOE_OK;
  if (int st = check_batch(C, table, max_pages, cache_len, new_off)) return st;
  if (!n_keep || (max_keep > 0 && !keep)) return MOE_ERR_ARG;
  if (!aligned_to(keep, 4) || !aligned_to(n_keep, 4) || !aligned_to(len_out, 4)) return MOE_ERR_ALIGN;
  if (len_out) {   // written by one workgroup of a sequence while others still read
    const int64_t bytes = 4 * static_cast<int64_t>(n_seqs);
    if (overlap(len_out, bytes, cache_len, bytes) || overlap(len_out, bytes, new_off, bytes + 4) ||
        overlap(len_out, bytes, n_keep, bytes) || overlap(len_out, bytes, keep, bytes * max_keep) ||
        overlap(len_out, bytes, table, bytes * max_pages) || over_cache(Rows{len_out, 1, bytes, bytes}, C))
      return MOE_ERR_ARG;
  }
  const KeepArgs a{batch_of(C, table, max_pages, cache_len, n_seqs, new_off, INT32_MAX, INT32_MAX, status),
                   C->k, C->v, C->k_scale, C->v_scale, keep, n_keep, len_out, max_keep};
  hipStream_t s = static_cast<hipStream_t>(stream);
  const dim3 grid(n_seqs, C->n_heads), block(256);
  if (C->head_dim == 64) hipLaunchKernelGGL(keep_kernel<64>, grid, block, 0, s, a);
  else if (C->head_dim == 128) hipLaunchKernelGGL(keep_kernel<128>, grid, block, 0, s, a);
  else hipLaunchKernelGGL(keep_kernel<256>, grid, block, 0, s, a);
  return launch_status(s);
}
