// attend.hip -- moe_tree_attention: softmax(scale q k) v of drafted tokens over a
// paged cache, each token seeing the cached tokens and the drafts its mask names.
#include "cache.hpp"

namespace moe {
namespace cache {
namespace {

struct AttendArgs {
  Batch b;
  const void *q, *kc, *vc;
  void* out;
  const uint64_t* mask;
  int64_t ld_q, ld_out;
  float scale;
  int n_q_heads, mask_words;
};

// One wave per new token and query head: the keys one after another with a running
// maximum m and sum l, lanes over the head's channels.
template <int TYPE, int D>
__global__ void __launch_bounds__(kWave) attend_kernel(AttendArgs a) {
  typedef elem_t<TYPE> E;
  const int s = blockIdx.z, h = blockIdx.y, i = blockIdx.x, lane = threadIdx.x;
  bool ok;
  const Seq q = sequence(a.b, s, ok);
  if (!ok && lane == 0) report(a.b, MOE_ERR_SLOT);
  if (i >= q.n) return;
  const int64_t t = q.off + i;
  const int g = h / (a.n_q_heads / a.b.n_heads), P = 1 << a.b.page_shift;
  float qv[D / kWave], acc[D / kWave], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int c = 0; c < D / kWave; c++) {
    qv[c] = static_cast<float>(static_cast<const E*>(a.q)[t * a.ld_q + h * D + c * kWave + lane]);
    acc[c] = 0.f;
  }
  for (int j = 0; j < q.len + q.n; j++) {
    if (j >= q.len) {
      const int d = j - q.len;
      if (a.mask ? d >= 64 * a.mask_words || !(a.mask[t * a.mask_words + d / 64] >> (d % 64) & 1) : d > i) continue;
    }
    const int page = page_of(a.b, s, j);
    if (page < 0) {
      if (lane == 0) report(a.b, MOE_ERR_SLOT);
      continue;
    }
    const int64_t head = (static_cast<int64_t>(page) * a.b.n_heads + g) * D * P;
    const int o = j & (P - 1);
    float x = 0.f;
#pragma unroll
    for (int c = 0; c < D / kWave; c++)
      x = __fmaf_rn(qv[c], static_cast<float>(static_cast<const E*>(a.kc)[head + o * D + c * kWave + lane]), x);
    for (int w = 32; w; w >>= 1) x += __shfl_xor(x, w);
    x *= a.scale;
    const float m2 = x > m ? x : m;
    const float keep = m2 == m ? 1.f : __expf(m - m2), p = x == -INFINITY ? 0.f : __expf(x - m2);
    l = l * keep + p;
#pragma unroll
    for (int c = 0; c < D / kWave; c++)
      acc[c] = acc[c] * keep + p * static_cast<float>(static_cast<const E*>(a.vc)[head + (c * kWave + lane) * P + o]);
    m = m2;
  }
#pragma unroll
  for (int c = 0; c < D / kWave; c++)
    static_cast<E*>(a.out)[t * a.ld_out + h * D + c * kWave + lane] = static_cast<E>(l == 0.f ? 0.f : acc[c] / l);
}

template <int TYPE>
void launch(int head_dim, dim3 grid, hipStream_t s, const AttendArgs& a) {
  if (head_dim == 64) hipLaunchKernelGGL((attend_kernel<TYPE, 64>), grid, dim3(kWave), 0, s, a);
  else if (head_dim == 128) hipLaunchKernelGGL((attend_kernel<TYPE, 128>), grid, dim3(kWave), 0, s, a);
  else hipLaunchKernelGGL((attend_kernel<TYPE, 256>), grid, dim3(kWave), 0, s, a);
}

int check_sizes(const moe_cache_t* C, int32_t n_q_heads, int32_t n_seqs, int32_t max_new, int32_t max_len) {
  if (int st = check_cache(C)) return st;
  if (n_seqs < 0 || n_seqs > 65535 || max_new < 0 || max_len < 0) return MOE_ERR_ARG;
  if (n_q_heads < 1 || n_q_heads > 65535 || n_q_heads % C->n_heads || n_q_heads / C->n_heads > 64) return MOE_ERR_ARG;
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
  if (n_split) *n_split = 1;
  if (ws_bytes) *ws_bytes = 0;
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
  const AttendArgs a{batch_of(C, table, max_pages, cache_len, n_seqs, new_off, n_tokens, max_new, status),
                     q, C->k, C->v, out, mask, ld_q, ld_out, scale, n_q_heads, mask_words};
  const dim3 grid(max_new, n_q_heads, n_seqs);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (C->type == MOE_TYPE_BF16) launch<MOE_TYPE_BF16>(C->head_dim, grid, s, a);
  else launch<MOE_TYPE_FP16>(C->head_dim, grid, s, a);
  return launch_status(s);
}
