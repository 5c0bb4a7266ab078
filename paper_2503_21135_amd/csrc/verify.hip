// verify.hip -- moe_draft_verify: which drafted tokens a model accepts, and the token after
// them, from given random numbers.
//
// Whether a draft is accepted, once the walk stands at its parent and has refused its elder
// siblings, does not depend on the rest of the walk: so every draft is tested at once, and the
// walk follows the answers.  Four steps:
//   stats_kernel    per row and chunk of the vocabulary: maximum, first index of it, sum of
//                   exponentials                                    (reads every logit once)
//   level_kernel    trees with draft probabilities: per row the sums that remain after each
//                   refused sibling but the last
//   walk_kernel     per sequence: the tests, the walk, keep, and what is drawn from
//   total_kernel    per sequence and chunk: the sum of what remains at the walk's end, 64 bits
//   pick_kernel     per sequence: the chunk, and the token in it, that u_next falls on
#include <algorithm>

#include "elem.hpp"

namespace moe {
namespace verify {
namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 4096;        // tokens of the vocabulary of a workgroup
constexpr int kEach = kChunk / kThreads;
constexpr int kMaxNew = 1024;

struct Args {
  const void *logits, *draft;
  const int32_t *tokens, *parents, *off;
  const float *temperature, *u, *u_next;
  int32_t *keep, *n_keep, *next, *status;
  double *sum, *level, *total;   // [n_tokens][chunks], [n_tokens], [n_seqs][chunks]
  float* top;                    // [n_tokens][chunks]
  int32_t *arg, *end;            // [n_tokens][chunks], [n_seqs]: the walk's last row, -1: nothing to draw
  double *row_sum;               // [n_tokens]: of each row, and its maximum
  float *row_top;
  int64_t ld, ld_draft;
  int n_seqs, n_tokens, max_new, vocab, chunks, type, draft_type;
};

struct Seq { int off, n; };

__device__ __forceinline__ void report(const Args& a, int status) {
  if (a.status) *a.status = status;
}
__device__ __forceinline__ Seq sequence(const Args& a, int b, bool& ok) {
  Seq s{a.off[b], a.off[b + 1] - a.off[b]};
  ok = s.n >= 0 && s.n <= a.max_new && s.off >= 0 && s.off <= a.n_tokens - s.n;
  if (!ok) s = Seq{0, 0};
  return s;
}
__device__ __forceinline__ float heat_of(const Args& a, int b) { return a.temperature ? a.temperature[b] : 1.f; }
__device__ __forceinline__ bool greedy(const Args& a, int b) { return !a.u || heat_of(a, b) == 0.f; }

// 16 consecutive logits or probabilities from any aligned address, past the end -inf
template <int TYPE>
__device__ __forceinline__ void load16(const void* base, int64_t at, int left, float fill, float (&x)[kEach]) {
  typedef elem_t<TYPE> E;
  struct __attribute__((packed, aligned(sizeof(E)))) Piece { E e[16 / sizeof(E)]; };
  constexpr int N = 16 / sizeof(E);
  const E* p = static_cast<const E*>(base) + at;
  if (left >= kEach) {
#pragma unroll
    for (int i = 0; i < kEach / N; i++) {
      const Piece w = reinterpret_cast<const Piece*>(p)[i];
#pragma unroll
      for (int e = 0; e < N; e++) x[i * N + e] = static_cast<float>(w.e[e]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kEach; i++) x[i] = i < left ? static_cast<float>(p[i]) : fill;
  }
}
__device__ __forceinline__ void load16(int type, const void* base, int64_t at, int left, float fill, float (&x)[kEach]) {
  if (type == MOE_TYPE_FP32) load16<MOE_TYPE_FP32>(base, at, left, fill, x);
  else if (type == MOE_TYPE_BF16) load16<MOE_TYPE_BF16>(base, at, left, fill, x);
  else load16<MOE_TYPE_FP16>(base, at, left, fill, x);
}

// exp(d / heat) for d <= 0, the argument's rounding errors taken along
struct Exp {
  float hi, lo;   // log2(e) / heat
  __device__ explicit Exp(float heat) {
    const double c = fmin(1.4426950408889634 / static_cast<double>(heat), 1e30);
    hi = static_cast<float>(c);
    lo = static_cast<float>(c - hi);
  }
  __device__ float operator()(float d) const {
    const float t = d * hi, e = __builtin_amdgcn_exp2f(t);
    const float r = __fmaf_rn(e, (__fmaf_rn(d, hi, -t) + d * lo) * 0.69314718f, e);
    return t < -120.f ? 0.f : r;
  }
};

__device__ __forceinline__ double wave_sum64(double v) {
  for (int w = 32; w; w >>= 1) v += __shfl_xor(v, w);
  return v;
}

__global__ void __launch_bounds__(kThreads) stats_kernel(Args a) {
  __shared__ float tops[kThreads / kWave];
  __shared__ int args[kThreads / kWave];
  __shared__ double sums[kThreads / kWave];
  const int chunk = blockIdx.x, i = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  bool ok;
  const Seq s = sequence(a, b, ok);
  if (i >= s.n) return;
  const int64_t row = s.off + i;
  const int at = chunk * kChunk + tid * kEach;
  float x[kEach];
  load16(a.type, a.logits, row * a.ld + at, a.vocab - at, -INFINITY, x);
  float top = -INFINITY;
  int arg = 0;
  bool nan = false;
#pragma unroll
  for (int e = 0; e < kEach; e++) {
    nan = nan || x[e] != x[e];
    if (x[e] > top) {
      top = x[e];
      arg = at + e;
    }
  }
  for (int w = 32; w; w >>= 1) {
    const float t = __shfl_xor(top, w);
    const int g = __shfl_xor(arg, w);
    if (t > top || (t == top && g < arg)) {
      top = t;
      arg = g;
    }
  }
  if (tid % kWave == 0) {
    tops[tid / kWave] = top;
    args[tid / kWave] = arg;
  }
  __syncthreads();
  for (int w = 0; w < kThreads / kWave; w++)
    if (tops[w] > top || (tops[w] == top && args[w] < arg)) {
      top = tops[w];
      arg = args[w];
    }
  double sum = 0.;
  if (!greedy(a, b)) {
    const Exp ex(heat_of(a, b));
    const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int e = 0; e < kEach; e++) sum += static_cast<double>(ex(x[e] - base));
  }
  if (nan) sum = __builtin_nan("");
  sum = wave_sum64(sum);
  if (tid % kWave == 0) sums[tid / kWave] = sum;
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < kThreads / kWave; w++) sum += sums[w];
    a.top[row * a.chunks + chunk] = top;
    a.arg[row * a.chunks + chunk] = arg;
    a.sum[row * a.chunks + chunk] = sum;
  }
}

// A row's probability of a token, in 64 bits.
__device__ __forceinline__ double prob(const Args& a, double x, float top, double sum, double heat) {
  return exp((x - top) / heat) / sum;
}

// what remains of p after the refused siblings whose sums are in `levels`, n of them; a sum of 0
// refused nothing
__device__ __forceinline__ double remains(double p, double d, const double* levels, int n) {
  double r = p, z = 1.;
  for (int k = 0; k < n; k++) {
    if (levels[k] == 0.) continue;
    r = fmax(r / z - d, 0.);
    z = levels[k];
  }
  return r / z;
}

// combines a row's chunks: all lanes of a wave get the maximum, its first index and the sum
__device__ __forceinline__ void join_row(const Args& a, int64_t row, Exp ex, int lane, float& top, int& arg, double& sum) {
  top = -INFINITY;
  arg = 0;
  for (int c = lane; c < a.chunks; c += kWave) {
    const float t = a.top[row * a.chunks + c];
    if (t > top) {
      top = t;
      arg = a.arg[row * a.chunks + c];
    }
  }
  for (int w = 32; w; w >>= 1) {
    const float t = __shfl_xor(top, w);
    const int g = __shfl_xor(arg, w);
    if (t > top || (t == top && g < arg)) {
      top = t;
      arg = g;
    }
  }
  sum = 0.;
  for (int c = lane; c < a.chunks; c += kWave) {
    const float t = a.top[row * a.chunks + c];
    sum += a.sum[row * a.chunks + c] * (t == top ? 1. : t == -INFINITY ? 1. : static_cast<double>(ex(t - top)));
  }
  sum = wave_sum64(sum);
}

// Per row: its own statistics, and for trees with draft probabilities the level sums.
__global__ void __launch_bounds__(kThreads) level_kernel(Args a) {
  __shared__ int kids[kMaxNew], n_kids;
  __shared__ double levels[kMaxNew], parts[kThreads / kWave];
  const int i = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
  bool ok;
  const Seq s = sequence(a, b, ok);
  if (i >= s.n || greedy(a, b)) return;
  if (tid == 0) {   // drafts below row i, in order
    int n = 0;
    for (int j = i + 1; j < s.n; j++)
      if (a.parents[s.off + j] == i && a.tokens[s.off + j] >= 0 && a.tokens[s.off + j] < a.vocab) kids[n++] = j;
    n_kids = n;
  }
  __syncthreads();
  if (n_kids < 2) return;
  const int64_t row = s.off + i;
  const float heat = heat_of(a, b);
  if (!(heat > 0.f) || heat == INFINITY) return;
  float top;
  int arg;
  double sum;
  join_row(a, row, Exp(heat), tid % kWave, top, arg, sum);
  for (int k = 0; k + 1 < n_kids; k++) {
    double z = 1.;
    for (int e = 0; e < k; e++) z = levels[e] == 0. ? z : levels[e];
    double total = 0.;
    for (int at = tid * kEach; at < a.vocab; at += kThreads * kEach) {
      float x[kEach], d[kEach];
      load16(a.type, a.logits, row * a.ld + at, a.vocab - at, -INFINITY, x);
      load16(a.draft_type, a.draft, row * a.ld_draft + at, a.vocab - at, 0.f, d);
#pragma unroll
      for (int e = 0; e < kEach; e++)
        total += fmax(remains(prob(a, x[e], top, sum, heat), d[e], levels, k) - static_cast<double>(d[e]), 0.);
    }
    total = wave_sum64(total);
    if (tid % kWave == 0) parts[tid / kWave] = total;
    __syncthreads();
    if (tid == 0) {
      levels[k] = ((parts[0] + parts[1]) + parts[2]) + parts[3];
      a.level[s.off + kids[k]] = levels[k];
    }
    __syncthreads();
  }
}

__global__ void __launch_bounds__(kThreads) walk_kernel(Args a) {
  __shared__ double sums[kMaxNew];
  __shared__ float tops[kMaxNew];
  __shared__ int args[kMaxNew], parent[kMaxNew], token[kMaxNew];
  __shared__ uint8_t yes[kMaxNew];
  __shared__ int path[kMaxNew], n_path, last;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid % kWave;
  bool ok;
  const Seq s = sequence(a, b, ok);
  if (!ok && tid == 0) report(a, MOE_ERR_SLOT);
  const float heat = heat_of(a, b);
  const bool first = greedy(a, b), cold = !first && (!(heat > 0.f) || heat == INFINITY);
  const Exp ex(heat);
  for (int i = tid / kWave; i < s.n; i += kThreads / kWave) {
    float top;
    int arg;
    double sum;
    join_row(a, s.off + i, ex, lane, top, arg, sum);
    // not a distribution: NaN for a sum
    if (cold || !(__builtin_fabsf(top) < INFINITY)) sum = __builtin_nan("");
    if (lane == 0) {
      sums[i] = sum;
      tops[i] = top;
      args[i] = arg;
      a.row_sum[s.off + i] = sum;
      a.row_top[s.off + i] = top;
    }
  }
  for (int i = tid; i < s.n; i += kThreads) {
    int p = i ? (a.parents ? a.parents[s.off + i] : i - 1) : -1;
    const int x = a.tokens[s.off + i];
    if (i && (p < -1 || p >= i || x < 0 || x >= a.vocab)) {
      report(a, MOE_ERR_SLOT);
      p = -1;
    }
    parent[i] = p;
    token[i] = x;
  }
  __syncthreads();
  for (int i = tid; i < s.n; i += kThreads) {
    const int p = parent[i], x = token[i];
    bool accepted = false;
    if (p >= 0 && sums[p] == sums[p]) {
      if (first) {
        accepted = args[p] == x;
      } else {
        const float un = fminf(fmaxf(a.u[s.off + i], 0.f), 0x1.fffffep-1f);
        const double pr = prob(a, load_elem(a.logits, (s.off + p) * a.ld + x, a.type), tops[p], sums[p], heat);
        if (a.draft) {
          const double d = load_elem(a.draft, (s.off + p) * a.ld_draft + x, a.draft_type);
          double r = pr, z = 1.;   // with the sums after the elder siblings
          for (int j = p + 1; j < i; j++)
            if (parent[j] == p) {
              const double level = a.level[s.off + j];
              if (level == 0.) continue;
              r = fmax(r / z - d, 0.);
              z = level;
            }
          accepted = un * d < r / z;
        } else {
          double left = 1.;   // without the elder siblings
          bool again = false;
          for (int j = p + 1; j < i; j++)
            if (parent[j] == p) {
              bool seen = false;
              for (int e = p + 1; e < j; e++) seen = seen || (parent[e] == p && token[e] == token[j]);
              again = again || token[j] == x;
              if (!seen) left -= prob(a, load_elem(a.logits, (s.off + p) * a.ld + token[j], a.type), tops[p], sums[p], heat);
            }
          accepted = !again && un * left < pr;
        }
      }
    }
    yes[i] = accepted;
  }
  __syncthreads();
  if (tid == 0) {
    int n = 0, cur = 0;
    if (s.n > 0) path[n++] = 0;
    for (int i = 1; i < s.n; i++)
      if (parent[i] == cur && yes[i]) path[n++] = cur = i;
    const bool none = s.n > 0 && sums[cur] != sums[cur];
    if (none) report(a, MOE_ERR_RANGE);
    n_path = n;
    a.n_keep[b] = n;
    a.end[b] = s.n == 0 || none || first ? -1 : cur;
    if (s.n == 0 || none) a.next[b] = -1;
    else if (first) a.next[b] = args[cur];
  }
  __syncthreads();
  for (int j = tid; j < a.max_new; j += kThreads) a.keep[static_cast<int64_t>(b) * a.max_new + j] = j < n_path ? path[j] : -1;
}

// What there is to draw from at the end of a walk.
struct Rest {
  int64_t row;
  int n;         // refused drafts
  float top;
  double sum, heat;
};
struct RestLds {
  int token[kMaxNew];
  double level[kMaxNew];
  int n;
};

__device__ __forceinline__ Rest rest_of(const Args& a, int b, const Seq& s, int cur, RestLds& lds, int tid) {
  Rest r;
  r.row = s.off + cur;
  r.top = a.row_top[r.row];
  r.sum = a.row_sum[r.row];
  r.heat = heat_of(a, b);
  if (tid == 0) {
    int n = 0;
    for (int j = cur + 1; j < s.n; j++) {
      const int p = a.parents ? a.parents[s.off + j] : j - 1, x = a.tokens[s.off + j];
      if (p != cur || x < 0 || x >= a.vocab) continue;
      lds.token[n] = x;
      lds.level[n++] = a.draft && a.parents ? a.level[s.off + j] : 0.;   // not set for the last one
    }
    lds.n = n;
  }
  __syncthreads();
  r.n = lds.n;
  return r;
}

// 16 tokens' shares from `at` on, after `n` refusals
__device__ __forceinline__ void shares(const Args& a, const Rest& r, const RestLds& lds, int n, int at, double (&v)[kEach]) {
  float x[kEach];
  load16(a.type, a.logits, r.row * a.ld + at, a.vocab - at, -INFINITY, x);
#pragma unroll
  for (int e = 0; e < kEach; e++) v[e] = exp((static_cast<double>(x[e]) - r.top) / r.heat);
  if (n == 0) return;
  if (a.draft) {
    float d[kEach];
    load16(a.draft_type, a.draft, r.row * a.ld_draft + at, a.vocab - at, 0.f, d);
#pragma unroll
    for (int e = 0; e < kEach; e++) v[e] = fmax(remains(v[e] / r.sum, d[e], lds.level, n - 1) - static_cast<double>(d[e]), 0.);
  } else {
    for (int k = 0; k < n; k++) {
      const int e0 = lds.token[k] - at;
#pragma unroll
      for (int e = 0; e < kEach; e++) v[e] = e == e0 ? 0. : v[e];
    }
  }
}

__device__ __forceinline__ double block_sum(double v, double* parts, int tid) {
  v = wave_sum64(v);
  __syncthreads();
  if (tid % kWave == 0) parts[tid / kWave] = v;
  __syncthreads();
  return ((parts[0] + parts[1]) + parts[2]) + parts[3];
}

__global__ void __launch_bounds__(kThreads) total_kernel(Args a) {
  __shared__ RestLds lds;
  __shared__ double parts[kThreads / kWave];
  const int chunk = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
  const int cur = a.end[b];
  if (cur < 0) return;
  bool ok;
  const Seq s = sequence(a, b, ok);
  const Rest r = rest_of(a, b, s, cur, lds, tid);
  double v[kEach];
  shares(a, r, lds, r.n, chunk * kChunk + tid * kEach, v);
  double t = 0.;
#pragma unroll
  for (int e = 0; e < kEach; e++) t += v[e];
  t = block_sum(t, parts, tid);
  if (tid == 0) a.total[static_cast<int64_t>(b) * a.chunks + chunk] = t;
}

__global__ void __launch_bounds__(kThreads) pick_kernel(Args a) {
  __shared__ RestLds lds;
  __shared__ double parts[kThreads / kWave], sums[kThreads];
  __shared__ int found;
  const int b = blockIdx.x, tid = threadIdx.x;
  const int cur = a.end[b];
  if (cur < 0) return;
  bool ok;
  const Seq s = sequence(a, b, ok);
  const Rest r = rest_of(a, b, s, cur, lds, tid);
  double* total = a.total + static_cast<int64_t>(b) * a.chunks;
  int n = r.n;
  double all;
  for (;;) {
    double t = 0.;
    for (int c = tid; c < a.chunks; c += kThreads) t += total[c];
    all = block_sum(t, parts, tid);
    if (all > 0. || n == 0) break;
    n--;    // nothing remains after the last refusal: what there was before it
    for (int c = 0; c < a.chunks; c++) {
      double v[kEach], sum = 0.;
      shares(a, r, lds, n, c * kChunk + tid * kEach, v);
#pragma unroll
      for (int e = 0; e < kEach; e++) sum += v[e];
      sum = block_sum(sum, parts, tid);
      if (tid == 0) total[c] = sum;
    }
    __syncthreads();
  }
  const double aim = static_cast<double>(fminf(fmaxf(a.u_next[b], 0.f), 0x1.fffffep-1f)) * all;
  // the chunk: the first whose end passes the aim, or the last that has anything
  if (tid == 0) {
    double up = 0., before = 0.;
    int at = 0;
    for (int c = 0; c < a.chunks; c++) {
      const double t = total[c];
      if (t > 0.) {
        at = c;
        before = up;
      }
      up += t;
      if (up > aim) break;
    }
    found = at;
    parts[0] = before;
  }
  __syncthreads();
  const int at = found * kChunk + tid * kEach;
  const double before = parts[0];
  double v[kEach], sum = 0.;
  shares(a, r, lds, n, at, v);
#pragma unroll
  for (int e = 0; e < kEach; e++) sum += v[e];
  sums[tid] = sum;
  __syncthreads();
  if (tid == 0) {
    double up = before, mine = before;
    int t = 0;
    for (int i = 0; i < kThreads; i++) {
      if (sums[i] > 0.) {
        t = i;
        mine = up;
      }
      up += sums[i];
      if (up > aim) break;
    }
    found = t;
    parts[0] = mine;
  }
  __syncthreads();
  if (tid == found) {
    double up = parts[0];
    int x = 0;
    bool done = false;
#pragma unroll
    for (int e = 0; e < kEach; e++) {
      if (!done && v[e] > 0.) x = e;
      up += v[e];
      done = done || up > aim;
    }
    a.next[b] = at + x;
  }
}

struct Layout {
  int64_t chunks;
  size_t sum, level, row_sum, total, top, row_top, arg, end, bytes;
};
Layout layout_of(int64_t n_seqs, int64_t n_tokens, int64_t vocab) {
  Layout l;
  l.chunks = cdiv(vocab, kChunk);
  size_t at = 0;
  auto put = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 15) / 16 * 16;
    return here;
  };
  l.sum = put(8 * n_tokens * l.chunks);
  l.level = put(8 * n_tokens);
  l.row_sum = put(8 * n_tokens);
  l.total = put(8 * n_seqs * l.chunks);
  l.top = put(4 * n_tokens * l.chunks);
  l.row_top = put(4 * n_tokens);
  l.arg = put(4 * n_tokens * l.chunks);
  l.end = put(4 * n_seqs);
  l.bytes = at;
  return l;
}

int check_sizes(int32_t n_seqs, int32_t n_tokens, int32_t max_new, int32_t vocab) {
  if (n_seqs < 0 || n_seqs > 65535 || n_tokens < 0 || max_new < 0 || max_new > kMaxNew || vocab < 1 || vocab > (1 << 28)) return MOE_ERR_ARG;
  return MOE_OK;
}

}  // namespace
}  // namespace verify
}  // namespace moe

extern "C" int moe_draft_verify_plan(int32_t n_seqs, int32_t n_tokens, int32_t max_new, int32_t vocab, size_t* ws_bytes) {
  using namespace moe::verify;
  if (int st = check_sizes(n_seqs, n_tokens, max_new, vocab)) return st;
  if (ws_bytes) *ws_bytes = layout_of(n_seqs, n_tokens, vocab).bytes;
  return MOE_OK;
}

extern "C" int moe_draft_verify(const void* logits, int32_t logits_type, int64_t ld_logits, int32_t n_tokens,
                                int32_t vocab, const int32_t* tokens, const int32_t* parents,
                                const int32_t* new_off, int32_t n_seqs, int32_t max_new,
                                const void* draft, int32_t draft_type, int64_t ld_draft,
                                const float* temperature, const float* u, const float* u_next,
                                int32_t* keep, int32_t* n_keep, int32_t* next, int32_t* status,
                                void* ws, size_t ws_bytes, void* stream) {
  using namespace moe;
  using namespace moe::verify;
  if (int st = check_sizes(n_seqs, n_tokens, max_new, vocab)) return st;
  if (n_seqs == 0) return MOE_OK;
  if (!valid_type(logits_type) || (draft && !valid_type(draft_type)) || ld_logits < vocab || (draft && ld_draft < vocab)) return MOE_ERR_ARG;
  if (!new_off || !n_keep || !next || (max_new > 0 && !keep) || !u != !u_next) return MOE_ERR_ARG;
  if (n_tokens > 0 && (!logits || !tokens)) return MOE_ERR_ARG;
  if (!aligned_to(logits, type_bytes(logits_type)) || (draft && !aligned_to(draft, type_bytes(draft_type))) || !aligned_to(tokens, 4) ||
      !aligned_to(parents, 4) || !aligned_to(new_off, 4) || !aligned_to(temperature, 4) || !aligned_to(u, 4) || !aligned_to(u_next, 4) ||
      !aligned_to(keep, 4) || !aligned_to(n_keep, 4) || !aligned_to(next, 4) || !aligned_to(status, 4))
    return MOE_ERR_ALIGN;
  const Layout l = layout_of(n_seqs, n_tokens, vocab);
  if (!ws || ws_bytes < l.bytes) return MOE_ERR_WORKSPACE;
  if (!aligned16(ws)) return MOE_ERR_ALIGN;
  const int64_t seqs = n_seqs, rows = n_tokens;
  const struct { const void* p; int64_t n; } outs[] = {{keep, 4 * seqs * max_new}, {n_keep, 4 * seqs}, {next, 4 * seqs}},
      ins[] = {{logits, rows ? ((rows - 1) * ld_logits + vocab) * type_bytes(logits_type) : 0},
               {draft, draft && rows ? ((rows - 1) * ld_draft + vocab) * type_bytes(draft_type) : 0},
               {tokens, 4 * rows}, {parents, 4 * rows}, {new_off, 4 * seqs + 4}, {temperature, 4 * seqs}, {u, 4 * rows}, {u_next, 4 * seqs},
               {ws, static_cast<int64_t>(l.bytes)}};
  for (int i = 0; i < 3; i++) {
    for (int j = 0; j < i; j++)
      if (overlap(outs[i].p, outs[i].n, outs[j].p, outs[j].n)) return MOE_ERR_ARG;
    for (const auto& in : ins)
      if (overlap(outs[i].p, outs[i].n, in.p, in.n)) return MOE_ERR_ARG;
  }
  char* w = static_cast<char*>(ws);
  auto part = [&](size_t at) { return static_cast<void*>(w + at); };
  const Args a{logits, draft, tokens, parents, new_off, temperature, u, u_next, keep, n_keep, next, status,
               static_cast<double*>(part(l.sum)), static_cast<double*>(part(l.level)), static_cast<double*>(part(l.total)),
               static_cast<float*>(part(l.top)), static_cast<int32_t*>(part(l.arg)), static_cast<int32_t*>(part(l.end)),
               static_cast<double*>(part(l.row_sum)), static_cast<float*>(part(l.row_top)), ld_logits, ld_draft,
               n_seqs, n_tokens, max_new, vocab, static_cast<int>(l.chunks), logits_type, draft_type};
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int most = std::min(max_new, n_tokens);
  const unsigned chunks = static_cast<unsigned>(l.chunks);
  if (most > 0) {
    hipLaunchKernelGGL(stats_kernel, dim3(chunks, most, n_seqs), dim3(kThreads), 0, s, a);
    if (draft && parents && u) hipLaunchKernelGGL(level_kernel, dim3(most, n_seqs), dim3(kThreads), 0, s, a);
  }
  hipLaunchKernelGGL(walk_kernel, dim3(n_seqs), dim3(kThreads), 0, s, a);
  if (most > 0 && u) {
    hipLaunchKernelGGL(total_kernel, dim3(chunks, n_seqs), dim3(kThreads), 0, s, a);
    hipLaunchKernelGGL(pick_kernel, dim3(n_seqs), dim3(kThreads), 0, s, a);
  }
  return launch_status(s);
}
