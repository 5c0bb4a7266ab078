// cache.hpp -- the paged key/value cache as its kernels see it: the batch of
// sequences, the lookup of a token's page, and the checks of their arguments.
#pragma once

#include "elem.hpp"

namespace moe {
namespace cache {

// a batch of sequences over one cache (device side)
struct Batch {
  const int32_t* table;
  const int32_t* len;
  const int32_t* off;
  int32_t* status;
  int max_pages, n_seqs, n_tokens, max_new;
  int n_pages, n_heads, page_shift;
};

struct Seq {
  int len;   // cached tokens
  int n;     // new tokens
  int off;   // row of the first new token
};

__device__ __forceinline__ void report(const Batch& b, int status) {
  if (b.status) *b.status = status;
}

// Sequence s, with what is out of range set to nothing: `ok` false when a length or a
// row range is not one the caller may have.
__device__ __forceinline__ Seq sequence(const Batch& b, int s, bool& ok) {
  Seq q{b.len[s], b.off[s + 1] - b.off[s], b.off[s]};
  ok = q.len >= 0 && q.n >= 0 && q.n <= b.max_new && q.off >= 0 && q.off <= b.n_tokens - q.n &&
       q.len <= INT32_MAX - 4096 - q.n;   // slot numbers rounded up to a tile stay ints
  if (!ok) q = Seq{0, 0, 0};
  return q;
}

// Page that holds slot `slot` of sequence s, or -1.
__device__ __forceinline__ int page_of(const Batch& b, int s, int slot) {
  const int i = slot >> b.page_shift;
  if (i >= b.max_pages) return -1;
  const int p = b.table[static_cast<int64_t>(s) * b.max_pages + i];
  return p >= 0 && p < b.n_pages ? p : -1;
}

inline int check_cache(const moe_cache_t* C) {
  if (!C || C->n_pages < 1 || C->n_heads < 1 || C->n_heads > 65535 || !valid_type16(C->type)) return MOE_ERR_ARG;
  if (C->head_dim != 64 && C->head_dim != 128 && C->head_dim != 256) return MOE_ERR_ARG;
  if (C->page_size < 32 || C->page_size > 1024 || (C->page_size & (C->page_size - 1))) return MOE_ERR_ARG;
  return MOE_OK;
}

// MOE_OK when the cache, the table and the batch's index arrays can be used.
inline int check_batch(const moe_cache_t* C, const int32_t* table, int32_t max_pages, const int32_t* len,
                       const int32_t* off) {
  if (!C->k || !C->v || !table || !len || !off || max_pages < 1) return MOE_ERR_ARG;
  if (!aligned16(C->k) || !aligned16(C->v) || !aligned_to(table, 4) || !aligned_to(len, 4) || !aligned_to(off, 4))
    return MOE_ERR_ALIGN;
  return MOE_OK;
}

// Whether rows that a call writes share a byte with the cache's keys or values.
inline bool over_cache(const Rows& out, const moe_cache_t* C) {
  const int64_t bytes = static_cast<int64_t>(C->n_pages) * C->n_heads * C->page_size * C->head_dim * 2;
  return overlap(out, Rows{C->k, 1, bytes, bytes}) || overlap(out, Rows{C->v, 1, bytes, bytes});
}

inline Batch batch_of(const moe_cache_t* C, const int32_t* table, int32_t max_pages, const int32_t* len,
                      int32_t n_seqs, const int32_t* off, int32_t n_tokens, int32_t max_new, int32_t* status) {
  return Batch{table, len, off, status, max_pages, n_seqs, n_tokens, max_new,
               C->n_pages, C->n_heads, __builtin_ctz(static_cast<unsigned>(C->page_size))};
}

}  // namespace cache
}  // namespace moe
