// cache.hip -- moe_cache_append and moe_cache_keep: the two calls that write the
// paged key/value cache.
#include <algorithm>

#include "cache.hpp"

namespace moe {
namespace cache {
namespace {

constexpr int kThreads = 256;
constexpr int kSlots = 64;   // slots of an append workgroup, aligned: whole 8-slot pieces of a value row
constexpr int kDirect = 16;  // up to so many new tokens of a tile, values go to their places without LDS
constexpr int kRowsKept = 32;   // rows a keep workgroup holds in registers at a time

struct AppendArgs {
  Batch b;
  const void *q, *k, *v;
  void *q_out, *kc, *vc;
  const int32_t* positions;
  const float *cos, *sin;
  int64_t ld_q, ld_k, ld_v, ld_q_out;
  int group, rot_dim, max_pos, interleaved;
};

// 16 bytes at any address of a 16-bit type's row (global accesses need no alignment)
struct __attribute__((packed, aligned(2))) Piece { uint32_t w[4]; };

// One workgroup per 64 aligned slots of a sequence and key/value head g: the head's new
// keys and its query heads turned and stored, its values turned over through LDS into
// the page's [channel][slot] rows, 8 slots to a store.  Bound by HBM where there are
// many tokens, each row being read and written once (8192 tokens of 32 + 2 x 8 heads of
// 128, 206 MB: 51 us, 4.0 TB/s), else by its four dependent loads (one token 5.0 us, 32
// trees of 16 to 32 tokens 11.9 us).  4 D threads give each thread one pair of chunks of
// one token: with 256, which take two passes at D = 128, the trees take 14.9 us, one token
// 7.6, the prompt 49.
template <int TYPE, int D>
__global__ void __launch_bounds__(4 * D) append_kernel(AppendArgs a) {
  typedef elem_t<TYPE> E;
  constexpr int kItems = D / 16;        // pairs of 8-channel chunks of a head
  __shared__ int64_t pages[kSlots / 32];            // start of the head in each of the tile's pages, or -1
  __shared__ int where[kSlots];                     // position of each slot's token, or -1: no token, or one to skip
  __shared__ uint32_t turned[D][kSlots / 2 + 1];    // values, two slots to a word
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
  if (tid < kSlots) {
    const int slot = slot0 + tid;
    const bool live = slot >= q.len && slot < end;
    const int pos = !live ? -1 : (a.positions ? a.positions[t0 + tid] : slot);
    const bool bad = live && a.cos && (pos < 0 || pos >= a.max_pos);
    where[tid] = live && !bad ? (a.cos ? pos : 0) : -1;
    bool lost = false;
    if (tid % 32 == 0) {
      const int page = slot < end && slot + 32 > q.len ? page_of(a.b, s, slot) : 0;
      lost = page < 0;
      pages[tid / 32] = lost ? -1 : (static_cast<int64_t>(page) * a.b.n_heads + g) * D * P + (slot & (P - 1));
    }
    if (bad || lost) report(a.b, MOE_ERR_SLOT);
  }
  __syncthreads();

  // values: each thread two slots by 8 channels, on their way while the keys and queries
  // are turned
  const int vc8 = tid % (D / 8) * 8, pair = tid / (D / 8);
  Piece val[2] = {};
#pragma unroll
  for (int e = 0; e < 2; e++)
    if (where[2 * pair + e] >= 0)
      val[e] = *reinterpret_cast<const Piece*>(static_cast<const E*>(a.v) + (t0 + 2 * pair + e) * a.ld_v + g * D + vc8);

  // keys and queries: each thread one token's pair of chunks, of every head of the group
  const int half = a.rot_dim / 2, j = tid % kItems, o = tid / kItems, pos = where[o];
  if (pos >= 0) {
    const int64_t t = t0 + o;
    const bool turn = a.cos && 16 * j < a.rot_dim;
    const bool split = turn && !a.interleaved;    // chunks half a rotation apart
    const int c0 = split ? 8 * j : 16 * j, c1 = split ? half + 8 * j : 16 * j + 8;
    float cs[16], sn[16];   // per channel pair: 8 used when the pair spans the chunks
    if (turn) {
      const int64_t at = static_cast<int64_t>(pos) * half + 8 * j;
#pragma unroll
      for (int e = 0; e < 8; e++) {
        cs[e] = a.cos[at + e];
        sn[e] = a.sin[at + e];
      }
    }
    auto turned_pair = [&](Piece& x, Piece& y) {
      if (!turn) return;
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const float xl = half_lo<TYPE>(x.w[e]), xh = half_hi<TYPE>(x.w[e]), yl = half_lo<TYPE>(y.w[e]), yh = half_hi<TYPE>(y.w[e]);
        if (split) {
          x.w[e] = pack2<TYPE>(__fmaf_rn(xl, cs[2 * e], -(yl * sn[2 * e])), __fmaf_rn(xh, cs[2 * e + 1], -(yh * sn[2 * e + 1])));
          y.w[e] = pack2<TYPE>(__fmaf_rn(xl, sn[2 * e], yl * cs[2 * e]), __fmaf_rn(xh, sn[2 * e + 1], yh * cs[2 * e + 1]));
        } else {
          x.w[e] = pack2<TYPE>(__fmaf_rn(xl, cs[e], -(xh * sn[e])), __fmaf_rn(xl, sn[e], xh * cs[e]));
          y.w[e] = pack2<TYPE>(__fmaf_rn(yl, cs[4 + e], -(yh * sn[4 + e])), __fmaf_rn(yl, sn[4 + e], yh * cs[4 + e]));
        }
      }
    };
    const E* kp = static_cast<const E*>(a.k) + t * a.ld_k + g * D;
    Piece kx = *reinterpret_cast<const Piece*>(kp + c0), ky = *reinterpret_cast<const Piece*>(kp + c1);
    constexpr int kHeads = 4;     // query heads whose loads are issued together
    for (int h0 = 0; h0 < (a.q ? a.group : 0); h0 += kHeads) {
      Piece x[kHeads], y[kHeads];
      const int64_t c = (static_cast<int64_t>(g) * a.group + h0) * D;
#pragma unroll
      for (int h = 0; h < kHeads; h++)
        if (h0 + h < a.group) {
          const E* qp = static_cast<const E*>(a.q) + t * a.ld_q + c + h * D;
          x[h] = *reinterpret_cast<const Piece*>(qp + c0);
          y[h] = *reinterpret_cast<const Piece*>(qp + c1);
        }
#pragma unroll
      for (int h = 0; h < kHeads; h++)
        if (h0 + h < a.group) {
          E* op = static_cast<E*>(a.q_out) + t * a.ld_q_out + c + h * D;
          turned_pair(x[h], y[h]);
          *reinterpret_cast<Piece*>(op + c0) = x[h];
          *reinterpret_cast<Piece*>(op + c1) = y[h];
        }
    }
    const int64_t page = pages[o / 32];
    if (page >= 0) {
      const int in_page = (slot0 + o) & (P - 1);
      E* out = static_cast<E*>(a.kc) + page - (in_page & -32) + static_cast<int64_t>(in_page) * D;
      turned_pair(kx, ky);
      *reinterpret_cast<Piece*>(out + c0) = kx;
      *reinterpret_cast<Piece*>(out + c1) = ky;
    }
  }

  // few tokens: straight to their places, two bytes at a time, which spares the barrier
  // and the way back (one token 5.0 us, through LDS 6.1); many: through LDS (the 8192 tokens
  // 51 us, straight 61)
  if (min(end, slot0 + kSlots) - max(q.len, slot0) <= kDirect) {
#pragma unroll
    for (int e = 0; e < 2; e++) {
      const int o = 2 * pair + e;
      const int64_t page = pages[o / 32];
      if (where[o] < 0 || page < 0) continue;
      uint16_t* out = static_cast<uint16_t*>(a.vc) + page + static_cast<int64_t>(vc8) * P + o % 32;
#pragma unroll
      for (int i = 0; i < 8; i++) out[static_cast<int64_t>(i) * P] = static_cast<uint16_t>(val[e].w[i / 2] >> 16 * (i & 1));
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; e++) {
    turned[vc8 + 2 * e][pair] = (val[0].w[e] & 0xFFFFu) | val[1].w[e] << 16;
    turned[vc8 + 2 * e + 1][pair] = val[0].w[e] >> 16 | (val[1].w[e] & 0xFFFF0000u);
  }
  __syncthreads();
  for (int i = tid; i < D * (kSlots / 8); i += 4 * D) {
    const int o = i % (kSlots / 8) * 8, c = i / (kSlots / 8);
    if (slot0 + o + 8 <= q.len || slot0 + o >= end) continue;
    const int64_t page = pages[o / 32];
    if (page < 0) continue;
    uint16_t* out = static_cast<uint16_t*>(a.vc) + page + static_cast<int64_t>(c) * P + o % 32;
    u32x4 w;
    bool all = true;
#pragma unroll
    for (int e = 0; e < 4; e++) {
      w[e] = turned[c][o / 2 + e];
      all = all && where[o + 2 * e] >= 0 && where[o + 2 * e + 1] >= 0;
    }
    if (all) {
      *reinterpret_cast<u32x4*>(out) = w;
    } else {
#pragma unroll
      for (int e = 0; e < 8; e++)
        if (where[o + e] >= 0) out[e] = static_cast<uint16_t>(w[e / 2] >> 16 * (e & 1));
    }
  }
}

struct KeepArgs {
  Batch b;
  void *kc, *vc;
  const int32_t *keep, *n_keep;
  int32_t* len_out;
  int max_keep;
};

// One workgroup per sequence and head.  Rows go 32 at a time through registers, all read
// before any is written; indices ascend, so no later row's source is written before
// it is read.  Rows that stay where they are are left alone.  The transposed values make
// a moved row touch head_dim cache lines, which is what bounds a large batch (256
// sequences of 8 heads of 128, 12.8 MB of rows: 16 to 19 us; one sequence 3.6 us); 8 rows side
// by side share those lines (with channels side by side: 24.7 us).
template <int D>
__global__ void __launch_bounds__(kThreads) keep_kernel(KeepArgs a) {
  constexpr int kVec = kRowsKept * (D / 8) / kThreads;     // 16-byte pieces of key rows per thread
  constexpr int kVals = kRowsKept * D / kThreads;          // values per thread: 8 rows side by side, whose
                                                           // slots of a channel share cache lines
  __shared__ int64_t from[kRowsKept], to[kRowsKept];       // head starts, from < 0: nothing to move
  __shared__ int from_slot[kRowsKept], to_slot[kRowsKept];
  const int s = blockIdx.x, h = blockIdx.y, tid = threadIdx.x;
  bool ok;
  const Seq q = sequence(a.b, s, ok);
  const int n = a.n_keep[s];
  const int32_t* list = a.keep + static_cast<int64_t>(s) * a.max_keep;
  ok = ok && n >= 0 && n <= a.max_keep;
  bool bad = false;
  for (int j = tid; ok && j < n; j += kThreads) bad = bad || list[j] < 0 || list[j] >= q.n || (j > 0 && list[j] <= list[j - 1]);
  ok = !__syncthreads_or(bad) && ok;
  if (tid == 0 && h == 0) {
    if (!ok) report(a.b, MOE_ERR_SLOT);
    if (a.len_out) a.len_out[s] = a.b.len[s] + (ok ? n : 0);
  }
  if (!ok) return;
  const int P = 1 << a.b.page_shift;
  uint16_t *kc = static_cast<uint16_t*>(a.kc), *vc = static_cast<uint16_t*>(a.vc);
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
          f = (static_cast<int64_t>(pf) * a.b.n_heads + h) * D * P;
          to[tid] = (static_cast<int64_t>(pt) * a.b.n_heads + h) * D * P;
          from_slot[tid] = fs & (P - 1);
          to_slot[tid] = ts & (P - 1);
        }
      }
      from[tid] = f;
    }
    __syncthreads();
    u32x4 key[kVec];
    uint16_t val[kVals];
#pragma unroll
    for (int i = 0; i < kVec; i++) {
      const int row = (tid + i * kThreads) / (D / 8), c = (tid + i * kThreads) % (D / 8) * 8;
      if (from[row] >= 0) key[i] = *reinterpret_cast<const u32x4*>(kc + from[row] + static_cast<int64_t>(from_slot[row]) * D + c);
    }
#pragma unroll
    for (int i = 0; i < kVals; i++) {
      const int row = tid % 8 + i % (kRowsKept / 8) * 8, c = tid / 8 + i / (kRowsKept / 8) * (kThreads / 8);
      if (from[row] >= 0) val[i] = vc[from[row] + static_cast<int64_t>(c) * P + from_slot[row]];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kVec; i++) {
      const int row = (tid + i * kThreads) / (D / 8), c = (tid + i * kThreads) % (D / 8) * 8;
      if (from[row] >= 0) *reinterpret_cast<u32x4*>(kc + to[row] + static_cast<int64_t>(to_slot[row]) * D + c) = key[i];
    }
#pragma unroll
    for (int i = 0; i < kVals; i++) {
      const int row = tid % 8 + i % (kRowsKept / 8) * 8, c = tid / 8 + i / (kRowsKept / 8) * (kThreads / 8);
      if (from[row] >= 0) vc[to[row] + static_cast<int64_t>(c) * P + to_slot[row]] = val[i];
    }
  }
}

template <int TYPE>
void launch_append(int head_dim, dim3 grid, hipStream_t s, const AppendArgs& a) {
  if (head_dim == 64) hipLaunchKernelGGL((append_kernel<TYPE, 64>), grid, dim3(4 * 64), 0, s, a);
  else if (head_dim == 128) hipLaunchKernelGGL((append_kernel<TYPE, 128>), grid, dim3(4 * 128), 0, s, a);
  else hipLaunchKernelGGL((append_kernel<TYPE, 256>), grid, dim3(4 * 256), 0, s, a);
}

}  // namespace
}  // namespace cache
}  // namespace moe

extern "C" int moe_cache_append(const moe_cache_t* C, const int32_t* table, int32_t max_pages,
                                const int32_t* cache_len, int32_t n_seqs, const int32_t* new_off,
                                int32_t n_tokens, int32_t max_new, const void* q, int64_t ld_q,
                                int32_t n_q_heads, const void* k, int64_t ld_k, const void* v,
                                int64_t ld_v, const int32_t* positions, const float* cos,
                                const float* sin, int32_t rot_dim, int32_t max_pos,
                                int32_t interleaved, void* q_out, int64_t ld_q_out, int32_t* status,
                                void* stream) {
  using namespace moe;
  using namespace moe::cache;
  if (int st = check_cache(C)) return st;
  if (n_seqs < 0 || n_seqs > 65535 || n_tokens < 0 || max_new < 0) return MOE_ERR_ARG;
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
      !aligned_to(sin, 4) || !aligned_to(positions, 4))
    return MOE_ERR_ALIGN;
  if (q) {
    const int64_t wide = 2 * static_cast<int64_t>(n_q_heads) * D, slim = 2 * static_cast<int64_t>(C->n_heads) * D;
    const Rows out{q_out, n_tokens, wide, 2 * ld_q_out};
    if ((q != q_out && overlap(out, Rows{q, n_tokens, wide, 2 * ld_q})) || overlap(out, Rows{k, n_tokens, slim, 2 * ld_k}) ||
        overlap(out, Rows{v, n_tokens, slim, 2 * ld_v}) || over_cache(out, C))
      return MOE_ERR_ARG;
  }
  const AppendArgs a{batch_of(C, table, max_pages, cache_len, n_seqs, new_off, n_tokens, max_new, status),
                     q, k, v, q_out, C->k, C->v, positions, cos, sin, ld_q, ld_k, ld_v, ld_q_out,
                     n_q_heads / C->n_heads, rot_dim, max_pos, interleaved};
  // aligned tiles that max_new slots can touch
  const dim3 grid(static_cast<unsigned>((static_cast<int64_t>(max_new) + kSlots - 2) / kSlots + 1), n_seqs, C->n_heads);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (C->type == MOE_TYPE_BF16) launch_append<MOE_TYPE_BF16>(D, grid, s, a);
  else launch_append<MOE_TYPE_FP16>(D, grid, s, a);
  return launch_status(s);
}

extern "C" int moe_cache_keep(const moe_cache_t* C, const int32_t* table, int32_t max_pages,
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
                   C->k, C->v, keep, n_keep, len_out, max_keep};
  hipStream_t s = static_cast<hipStream_t>(stream);
  const dim3 grid(n_seqs, C->n_heads), block(kThreads);
  if (C->head_dim == 64) hipLaunchKernelGGL(keep_kernel<64>, grid, block, 0, s, a);
  else if (C->head_dim == 128) hipLaunchKernelGGL(keep_kernel<128>, grid, block, 0, s, a);
  else hipLaunchKernelGGL(keep_kernel<256>, grid, block, 0, s, a);
  return launch_status(s);
}
