// cache.hip -- moe_cache_append and moe_cache_keep: the two calls that write the
// paged key/value cache.
#include "cache.hpp"

namespace moe {
namespace cache {
namespace {

struct AppendArgs {
  Batch b;
  const void *q, *k, *v;
  void *q_out, *kc, *vc;
  const int32_t* positions;
  const float *cos, *sin;
  int64_t ld_q, ld_k, ld_v, ld_q_out;
  int n_q_heads, head_dim, rot_dim, max_pos, interleaved;
};

// Rotation of a head's values c and its partner by row `pos` of the tables.
template <int TYPE>
__device__ __forceinline__ elem_t<TYPE> rotated(const AppendArgs& a, const elem_t<TYPE>* x, int c, int pos) {
  if (!a.cos || c >= a.rot_dim) return x[c];
  const int half = a.rot_dim / 2;
  const int i = a.interleaved ? c / 2 : c % half;
  const bool second = a.interleaved ? c & 1 : c >= half;
  const float u = static_cast<float>(x[a.interleaved ? 2 * i : i]);
  const float w = static_cast<float>(x[a.interleaved ? 2 * i + 1 : i + half]);
  const float cs = a.cos[static_cast<int64_t>(pos) * half + i], sn = a.sin[static_cast<int64_t>(pos) * half + i];
  return static_cast<elem_t<TYPE>>(second ? __fmaf_rn(u, sn, w * cs) : __fmaf_rn(u, cs, -(w * sn)));
}

// One workgroup per new token: its key and value heads, then its query heads.
template <int TYPE>
__global__ void __launch_bounds__(256) append_kernel(AppendArgs a) {
  typedef elem_t<TYPE> E;
  const int s = blockIdx.y;
  bool ok;
  const Seq q = sequence(a.b, s, ok);
  if (!ok && threadIdx.x == 0) report(a.b, MOE_ERR_SLOT);
  for (int i = blockIdx.x; i < q.n; i += gridDim.x) {
    const int64_t t = q.off + i;
    const int slot = q.len + i, page = page_of(a.b, s, slot), o = slot & ((1 << a.b.page_shift) - 1);
    const int pos = a.positions ? a.positions[t] : slot;
    const bool bad_pos = a.cos && (pos < 0 || pos >= a.max_pos);
    if ((page < 0 || bad_pos) && threadIdx.x == 0) report(a.b, MOE_ERR_SLOT);
    if (bad_pos) continue;
    const int D = a.head_dim, P = 1 << a.b.page_shift;
    if (page >= 0)
      for (int c = threadIdx.x; c < a.b.n_heads * D; c += 256) {
        const int h = c / D, d = c % D;
        const int64_t head = (static_cast<int64_t>(page) * a.b.n_heads + h) * D * P;
        static_cast<E*>(a.kc)[head + o * D + d] = rotated<TYPE>(a, static_cast<const E*>(a.k) + t * a.ld_k + h * D, d, pos);
        static_cast<E*>(a.vc)[head + d * P + o] = static_cast<const E*>(a.v)[t * a.ld_v + c];
      }
    if (!a.q) continue;
    for (int c0 = 0; c0 < a.n_q_heads * D; c0 += 256) {
      const int c = c0 + threadIdx.x;
      E x{};
      if (c < a.n_q_heads * D) x = rotated<TYPE>(a, static_cast<const E*>(a.q) + t * a.ld_q + c / D * D, c % D, pos);
      __syncthreads();   // q_out may be q: a head's values are all read before any is written
      if (c < a.n_q_heads * D) static_cast<E*>(a.q_out)[t * a.ld_q_out + c] = x;
    }
  }
}

struct KeepArgs {
  Batch b;
  void *kc, *vc;
  const int32_t *keep, *n_keep;
  int32_t* len_out;
  int max_keep, head_dim;
};

// One workgroup per sequence and head.  The indices ascend, so row j's source is
// never written before it is read: a thread moves its channels row by row.
__global__ void __launch_bounds__(256) keep_kernel(KeepArgs a) {
  const int s = blockIdx.x, h = blockIdx.y;
  bool ok;
  const Seq q = sequence(a.b, s, ok);
  const int n = a.n_keep[s];
  const int32_t* list = a.keep + static_cast<int64_t>(s) * a.max_keep;
  ok = ok && n >= 0 && n <= a.max_keep;
  for (int j = 0; ok && j < n; j++) ok = list[j] >= 0 && list[j] < q.n && (j == 0 || list[j] > list[j - 1]);
  if (threadIdx.x == 0 && h == 0) {
    if (!ok) report(a.b, MOE_ERR_SLOT);
    if (a.len_out) a.len_out[s] = a.b.len[s] + (ok ? n : 0);
  }
  if (!ok) return;
  const int D = a.head_dim, P = 1 << a.b.page_shift;
  uint16_t *kc = static_cast<uint16_t*>(a.kc), *vc = static_cast<uint16_t*>(a.vc);
  for (int c = threadIdx.x; c < D; c += 256)
    for (int j = 0; j < n; j++) {
      const int from = q.len + list[j], to = q.len + j;
      const int pf = page_of(a.b, s, from), pt = page_of(a.b, s, to);
      if (pf < 0 || pt < 0) {
        if (c == 0) report(a.b, MOE_ERR_SLOT);
        continue;
      }
      const int64_t hf = (static_cast<int64_t>(pf) * a.b.n_heads + h) * D * P, ht = (static_cast<int64_t>(pt) * a.b.n_heads + h) * D * P;
      const int of = from & (P - 1), ot = to & (P - 1);
      kc[ht + ot * D + c] = kc[hf + of * D + c];
      vc[ht + c * P + ot] = vc[hf + c * P + of];
    }
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
  if (!k || !v || ld_k < static_cast<int64_t>(C->n_heads) * D || ld_v < static_cast<int64_t>(C->n_heads) * D)
    return MOE_ERR_ARG;
  if (!q != !q_out) return MOE_ERR_ARG;
  if (q && (n_q_heads < 1 || ld_q < static_cast<int64_t>(n_q_heads) * D || ld_q_out < static_cast<int64_t>(n_q_heads) * D ||
            (q == q_out && ld_q != ld_q_out)))
    return MOE_ERR_ARG;
  if (!cos != !sin || (cos && (rot_dim < 2 || rot_dim % 2 || rot_dim > D || max_pos < 1))) return MOE_ERR_ARG;
  if (!aligned_to(q, 2) || !aligned_to(k, 2) || !aligned_to(v, 2) || !aligned_to(q_out, 2) || !aligned_to(cos, 4) ||
      !aligned_to(sin, 4) || !aligned_to(positions, 4))
    return MOE_ERR_ALIGN;
  const AppendArgs a{batch_of(C, table, max_pages, cache_len, n_seqs, new_off, n_tokens, max_new, status),
                     q, k, v, q_out, C->k, C->v, positions, cos, sin, ld_q, ld_k, ld_v, ld_q_out,
                     n_q_heads, D, rot_dim, max_pos, interleaved};
  const dim3 grid(max_new, n_seqs);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (C->type == MOE_TYPE_BF16) hipLaunchKernelGGL(append_kernel<MOE_TYPE_BF16>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(append_kernel<MOE_TYPE_FP16>, grid, dim3(256), 0, s, a);
  return launch_status(s);
}

extern "C" int moe_cache_keep(const moe_cache_t* C, const int32_t* table, int32_t max_pages,
                              const int32_t* cache_len, int32_t n_seqs, const int32_t* new_off,
                              const int32_t* keep, int32_t max_keep, const int32_t* n_keep,
                              int32_t* len_out, int32_t* status, void* stream) {
  using namespace moe;
  using namespace moe::cache;
  if (int st = check_cache(C)) return st;
  if (n_seqs < 0 || max_keep < 0) return MOE_ERR_ARG;
  if (n_seqs == 0) return MOE_OK;
  if (int st = check_batch(C, table, max_pages, cache_len, new_off)) return st;
  if (!n_keep || (max_keep > 0 && !keep) || len_out == cache_len) return MOE_ERR_ARG;
  if (!aligned_to(keep, 4) || !aligned_to(n_keep, 4) || !aligned_to(len_out, 4)) return MOE_ERR_ALIGN;
  const KeepArgs a{batch_of(C, table, max_pages, cache_len, n_seqs, new_off, INT32_MAX, INT32_MAX, status),
                   C->k, C->v, keep, n_keep, len_out, max_keep, C->head_dim};
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipLaunchKernelGGL(keep_kernel, dim3(n_seqs, C->n_heads), dim3(256), 0, s, a);
  return launch_status(s);
}
