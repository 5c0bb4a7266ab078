// verify.hip -- moe_draft_verify: which drafted tokens a model accepts, and the token after
// them, from given random numbers.
//
// With draft probabilities d, what is left of p after refusals is always max(p - c d, 0) over its
// sum S(c): a refusal turns (p - c d)+ / S into ((p - c d)+ / S - d)+ = (p - (c + S) d)+ / S, so c
// grows by S, from c = 0, S = 1.  One refusal costs one sum over a row, and its sums by chunk of
// the vocabulary are what the next token is drawn from if the walk ends there.  Without
// probabilities a refusal takes one token out, and nothing is summed before the end.
//   stats_kernel   per row and block of it: maximum and sum of exponentials, or the first of the
//                  largest                                      (reads every logit once)
//   walk_kernel    per sequence: rows' statistics, drafts' probabilities, the walk to its end or
//                  to the first sum that it needs
//   pass_kernel    per sequence and chunk of the vocabulary: that sum; the last workgroup of a
//                  sequence adds up and walks on, and at the end of the walk draws.  Launched once
//                  for chains and picked drafts, a few times for drawn trees; the last launch sees
//                  to the rest alone.  Where there are few blocks, each workgroup of the first pass
//                  begins the walk itself, and no walk_kernel is launched.
#include <algorithm>

#include "elem.hpp"

namespace moe {
namespace verify {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kMaxNew = 1024;
constexpr int kApart = 32;          // counters to a cache line of their own: the card takes one count a line at a time

// Where a sequence's walk stands.
struct State {
  double c, s;      // what is left of row cur's p: (p - c d)+ / s
  double sum;       // the row's sum and maximum
  float top;
  int cur, at;      // the row, and the last draft that was tested
  int count;        // kept rows
  int need;         // what a pass has to sum: nothing any more, a refusal, or what is drawn from
  int more;         // whether a refused draft has younger siblings
};
enum { kDone = 0, kRefusal = 1, kDraw = 2 };

struct Args {
  const void *logits, *draft;
  const int32_t *tokens, *parents, *off;
  const float *temperature, *u, *u_next;
  int32_t *keep, *n_keep, *next, *status;
  double *sum, *total, *row_sum, *prob;   // [n_tokens][blocks], [n_seqs][chunks], [n_tokens], [n_tokens]
  float *top, *row_top, *share;           // [n_tokens][blocks], [n_tokens], [n_tokens]
  int32_t *arg, *above;                   // [n_tokens][blocks], [n_tokens]: parents, -1 where not acceptable
  State* state;                           // [n_seqs]
  unsigned* arrived;                      // [n_seqs], kApart of them apart
  int64_t ld, ld_draft;
  int n_seqs, n_tokens, max_new, vocab, type, draft_type;
  int blocks, chunks;                     // of a row: of its statistics, and of a pass
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

// N values from `at` on, wherever they start; `fill` from `left` on
template <int TYPE, int N>
__device__ __forceinline__ void load_some(const void* base, int64_t at, int left, float fill, float (&x)[N]) {
  typedef elem_t<TYPE> E;
  constexpr int M = std::min<int>(16 / sizeof(E), N);
  struct __attribute__((packed, aligned(sizeof(E)))) Piece { E e[M]; };
  const E* p = static_cast<const E*>(base) + at;
  if (left >= N) {
#pragma unroll
    for (int i = 0; i < N / M; i++) {
      const Piece w = reinterpret_cast<const Piece*>(p)[i];
#pragma unroll
      for (int e = 0; e < M; e++) x[i * M + e] = static_cast<float>(w.e[e]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; i++) x[i] = i < left ? static_cast<float>(p[i]) : fill;
  }
}
template <int N>
__device__ __forceinline__ void load_some(int type, const void* base, int64_t at, int left, float fill, float (&x)[N]) {
  if (type == MOE_TYPE_FP32) load_some<MOE_TYPE_FP32>(base, at, left, fill, x);
  else if (type == MOE_TYPE_BF16) load_some<MOE_TYPE_BF16>(base, at, left, fill, x);
  else load_some<MOE_TYPE_FP16>(base, at, left, fill, x);
}

__device__ __forceinline__ double wave_sum64(double v) {
  for (int w = 32; w; w >>= 1) v += __shfl_xor(v, w);
  return v;
}
__device__ __forceinline__ float wave_max(float v) {
  v = fmaxf(v, dpp<0xB1>(v));
  v = fmaxf(v, dpp<0x4E>(v));
  v = fmaxf(v, dpp<0x141>(v));
  v = fmaxf(v, dpp<0x140>(v));
  return rows_max(v);
}
// log2(e) / heat, finite for the smallest
__device__ __forceinline__ float rate_of(float heat) { return fminf(1.44269504088896340736f / heat, 1e30f); }

// A term e^y of a row's sum is an fp32 exponential: its argument has three roundings of 2^-24 |y| (difference,
// rate, product) and the exponential one of 2^-23, as have the factors that bring waves and
// blocks to one maximum, whose exponents add up to |y|: 2^-22 (2 + |y|) of itself at most.  The terms are added in
// 64 bits (a thread's 16 or 32 in 32 bits moved sums by up to 5e-7; 64 chains of 7 27.1 us that way, 27.7 this way).
// Reads every logit once, all loads of a thread before the first is used: 16 trees of 31 over 131072
// fp32 (190 MB) 34.2 us, 5.5 TB/s; 64 chains of 7 over 32000 bf16 (27 MB) 10.8 us; one chain of 4
// 4.1, a launch and two rounds of loads.
template <int TYPE, int EACH>
__global__ void __launch_bounds__(kThreads) stats_kernel(Args a) {
  __shared__ float tops[kWaves];
  __shared__ double sums[kWaves];
  __shared__ int args[kWaves];
  const int block = blockIdx.x, i = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  bool ok;
  const Seq s = sequence(a, b, ok);
  const float heat = heat_of(a, b);
  if (block == 0 && i == 0 && tid == 0) a.arrived[static_cast<int64_t>(b) * kApart] = 0;
  if (i >= s.n) return;
  const bool greedy = !a.u || heat == 0.f;
  const int64_t row = s.off + i;
  // 16 bytes of a lane side by side
  constexpr int M = 16 / sizeof(elem_t<TYPE>), kPieces = EACH / M;
  float x[kPieces][M];
  const int at = block * (kThreads * EACH) + tid * M;
  const bool whole = (block + 1) * static_cast<int64_t>(kThreads * EACH) <= a.vocab;   // the loads need not wait for each other
#pragma unroll
  for (int p = 0; p < kPieces; p++)
    load_some<TYPE>(a.logits, row * a.ld + at + p * kThreads * M, whole ? M : a.vocab - at - p * kThreads * M, -INFINITY, x[p]);
  float top = -INFINITY;
#pragma unroll
  for (int p = 0; p < kPieces; p++)
#pragma unroll
    for (int e = 0; e < M; e++) top = fmaxf(top, x[p][e]);
  top = wave_max(top);
  double sum = 0.;
  int arg = INT32_MAX;
  if (greedy) {
    bool nan = false;
#pragma unroll
    for (int p = kPieces - 1; p >= 0; p--)
#pragma unroll
      for (int e = M - 1; e >= 0; e--) {
        nan = nan || x[p][e] != x[p][e];
        if (x[p][e] == top) arg = at + p * kThreads * M + e;
      }
    for (int w = 32; w; w >>= 1) arg = min(arg, __shfl_xor(arg, w));
    if (__any(nan)) sum = __builtin_nan("");
  } else {
    const float rate = rate_of(heat), base = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int p = 0; p < kPieces; p++)
#pragma unroll
      for (int e = 0; e < M; e++) sum += static_cast<double>(__builtin_amdgcn_exp2f((x[p][e] - base) * rate));
    sum = wave_sum64(sum);
  }
  if (tid % kWave == 0) {
    tops[tid / kWave] = top;
    sums[tid / kWave] = sum;
    args[tid / kWave] = arg;
  }
  __syncthreads();
  if (tid == 0) {
#pragma unroll
    for (int w = 1; w < kWaves; w++) top = fmaxf(top, tops[w]);
    sum = 0.;
    arg = INT32_MAX;
    const float rate = greedy ? 0.f : rate_of(heat);
#pragma unroll
    for (int w = 0; w < kWaves; w++) {
      // a wave that found nothing but -infinity has no part in the sum, or NaN
      sum += greedy || tops[w] == top || tops[w] == -INFINITY ? sums[w] : sums[w] * __builtin_amdgcn_exp2f((tops[w] - top) * rate);
      if (tops[w] == top) arg = min(arg, args[w]);
    }
    a.top[row * a.blocks + block] = top;
    a.sum[row * a.blocks + block] = sum;
    if (greedy) a.arg[row * a.blocks + block] = arg;
  }
}

// a row's probability of a logit, in 64 bits
__device__ __forceinline__ double prob(double x, float top, double sum, double heat) { return exp((x - top) / heat) / sum; }

// A sequence's drafts as the walk reads them, in LDS that is sized for the call's longest.
constexpr int kDraftBytes = 48;
constexpr int kOpen = INT32_MIN;   // of `next`: not decided
struct Drafts {
  double *prob, *sum;     // at the parent; the sum of its own row, NaN: no distribution
  float *share, *u, *top; // of the draft distribution at the parent; its own row's maximum
  int *above, *token, *arg, *path, *taken;   // parents; first of the largest; kept rows; refused tokens

  __device__ __forceinline__ Drafts(char* lds, int most) {
    prob = reinterpret_cast<double*>(lds);
    sum = prob + most;
    share = reinterpret_cast<float*>(sum + most);
    u = share + most;
    top = u + most;
    above = reinterpret_cast<int*>(top + most);
    token = above + most;
    arg = token + most;
    path = arg + most;
    taken = path + most;
  }
};

__device__ __forceinline__ float clamped(float u) { return fminf(fmaxf(u, 0.f), 0x1.fffffep-1f); }

// the first draft below row `cur` from `from` on, or -1; in one wave
__device__ __forceinline__ int child(const Drafts& d, int n, int cur, int from, int lane) {
  for (int j0 = from; j0 < n; j0 += kWave) {
    const uint64_t kids = __ballot(j0 + lane < n && d.above[j0 + lane] == cur);
    if (kids) return j0 + __builtin_ctzll(kids);
  }
  return -1;
}

// Walks on, in one wave: to the end, or to a refusal that needs a sum.  Rows that are kept go to `path`.
// A lane holds one of 64 drafts, whose index only grows, and whether it is accepted as the first that is
// tested below its parent is known for all of them at once, so that a step of a chain is a ballot and
// a few scalar instructions (the longest walks of 64 chains of 7 4.8 us with a draft read from LDS at a time, 3.2 this way).
__device__ __forceinline__ void walk(const Args& a, const Seq& s, const Drafts& d, State& st, int* path, int* next, int lane) {
  int above = -2, base = -1, from = st.at + 1;
  uint64_t first = 0, lost = 0;   // of the 64: accepted if no elder was refused; without a distribution
  bool elder = false;             // of cur's drafts, one was refused here
  for (;;) {
    if (from >= s.n) {
      st.need = kDraw;
      return;
    }
    if ((from & -kWave) != base) {
      base = from & -kWave;
      const int j = base + lane;
      bool yes = false, bad = false;
      above = -2;
      if (j < s.n) {
        above = d.above[j];
        const double p = d.prob[j], u = clamped(d.u[j]), w = a.draft ? d.share[j] : 1.;
        yes = u * w < p;
        bad = d.sum[j] != d.sum[j];
      }
      first = __ballot(yes);
      lost = __ballot(bad);
    }
    const uint64_t kids = __ballot(above == st.cur) & ~0ull << (from - base);
    if (!kids) {
      from = base + kWave;
      continue;
    }
    const int bit = __builtin_ctzll(kids), i = base + bit;
    st.at = i;
    from = i + 1;
    bool yes = first >> bit & 1;
    if (a.draft && (st.c != 0. || st.s != 1.)) {
      const double w = d.share[i];
      yes = clamped(d.u[i]) * w * st.s < d.prob[i] - st.c * w;
    } else if (!a.draft && elder) {
      // taken out before, by an elder sibling
      bool again = false;
      for (int j0 = st.cur + 1; j0 < i; j0 += kWave) {
        const int j = j0 + lane;
        again = again || (j < i && d.above[j] == st.cur && d.token[j] == d.token[i]);
      }
      again = __any(again);
      if (again) continue;
      yes = clamped(d.u[i]) * st.s < d.prob[i];
    }
    if (yes) {
      if (lane == 0) path[st.count] = i;
      st.cur = i;
      st.count++;
      st.c = 0.;
      st.s = 1.;
      elder = false;
      if (lost >> bit & 1) {   // nothing to go on with
        if (lane == 0) {
          report(a, MOE_ERR_RANGE);
          *next = -1;
        }
        st.need = kDone;
        return;
      }
    } else if (a.draft) {
      st.need = kRefusal;
      st.more = (kids & kids - 1) != 0 || child(d, s.n, st.cur, base + kWave, lane) >= 0;
      return;
    } else {
      st.s -= d.prob[i];
      elder = true;
    }
  }
}

// The walk's beginning, by a whole workgroup: statistics of the sequence's rows, its drafts'
// probabilities, and on to the first sum.  st, next and the drafts are in LDS.
__device__ __forceinline__ void begin(const Args& a, int b, const Seq& s, const Drafts& d, State* out, int* next, int tid, int threads) {
  const int lane = tid % kWave;
  const float heat = heat_of(a, b);
  const bool greedy = !a.u || heat == 0.f, cold = !(heat >= 0.f) || heat == INFINITY;   // cold: no temperature, greedy or not
  const float rate = greedy ? 0.f : rate_of(heat);
  for (int i = tid; i < s.n; i += threads) {
    int p = i ? (a.parents ? a.parents[s.off + i] : i - 1) : -1;
    const int x = a.tokens[s.off + i];
    if (i && (p < -1 || p >= i || x < 0 || x >= a.vocab)) {
      report(a, MOE_ERR_SLOT);
      p = -1;
    }
    d.above[i] = p;
    d.token[i] = x;
    d.u[i] = greedy ? 0.f : a.u[s.off + i];
    d.prob[i] = p < 0 || greedy ? 0. : load_elem(a.logits, (s.off + p) * a.ld + x, a.type);   // the logit, for now
    d.share[i] = p < 0 || greedy || !a.draft ? 0.f : load_elem(a.draft, (s.off + p) * a.ld_draft + x, a.draft_type);
  }
  // rows' blocks: `wide` lanes to a row, a power of two
  const int wide = a.blocks >= kWave ? kWave : 1 << (32 - __builtin_clz(a.blocks) - ((a.blocks & (a.blocks - 1)) == 0));
  for (int i0 = tid / kWave * (kWave / wide); i0 < s.n; i0 += threads / wide) {
    const int i = i0 + lane / wide, c0 = lane % wide;
    const bool live = i < s.n;
    const int64_t at = (s.off + i) * static_cast<int64_t>(a.blocks);
    const float t0 = live && c0 < a.blocks ? a.top[at + c0] : -INFINITY;
    const double z0 = live && c0 < a.blocks ? a.sum[at + c0] : 0.;
    float top = t0;
    for (int c = c0 + wide; live && c < a.blocks; c += wide) top = fmaxf(top, a.top[at + c]);
    for (int w = wide / 2; w; w >>= 1) top = fmaxf(top, __shfl_xor(top, w));
    auto part = [&](float t, double z) {
      return greedy || t == top || t == -INFINITY ? z : z * static_cast<double>(__builtin_amdgcn_exp2f((t - top) * rate));
    };
    double sum = part(t0, z0);
    int arg = greedy && live && c0 < a.blocks && t0 == top ? a.arg[at + c0] : INT32_MAX;
    for (int c = c0 + wide; live && c < a.blocks; c += wide) {
      const float t = a.top[at + c];
      sum += part(t, a.sum[at + c]);
      if (greedy && t == top) arg = min(arg, a.arg[at + c]);
    }
    for (int w = wide / 2; w; w >>= 1) {
      sum += __shfl_xor(sum, w);
      arg = min(arg, __shfl_xor(arg, w));
    }
    // not a distribution: NaN for a sum
    if (cold || !(__builtin_fabsf(top) < INFINITY)) sum = __builtin_nan("");
    if (live && c0 == 0) {
      d.sum[i] = sum;
      d.top[i] = top;
      d.arg[i] = arg;
    }
  }
  __syncthreads();
  if (!greedy) {
    for (int i = tid; i < s.n; i += threads) {
      const int p = d.above[i];
      if (p >= 0) d.prob[i] = prob(d.prob[i], d.top[p], d.sum[p], heat);
    }
    __syncthreads();
  }
  if (tid < kWave) {
    State st{0., 1., 0., 0.f, 0, 0, s.n > 0, kDone, 0};
    if (lane == 0) {
      *next = kOpen;
      if (s.n) d.path[0] = 0;
    }
    if (s.n == 0 || d.sum[0] != d.sum[0]) {
      if (lane == 0) {
        if (s.n) report(a, MOE_ERR_RANGE);
        *next = -1;
      }
    } else if (greedy) {
      // a lane's draft is its parent's largest or not; along the path as walk() goes
      bool none = false;
      for (int base = 0; base < s.n && !none; base += kWave) {
        const int j = base + lane, above = j > 0 && j < s.n ? d.above[j] : -1;
        const bool hit = above >= 0 && d.token[j] == d.arg[above];
        const uint64_t lost = __ballot(j < s.n && d.sum[j] != d.sum[j]);
        for (uint64_t kids; (kids = __ballot(hit && above == st.cur)) != 0;) {
          const int bit = __builtin_ctzll(kids);
          st.cur = base + bit;
          if (lane == 0) d.path[st.count] = st.cur;
          st.count++;
          none = lost >> bit & 1;
          if (none) break;
        }
      }
      if (lane == 0) {
        if (none) report(a, MOE_ERR_RANGE);
        *next = none ? -1 : d.arg[st.cur];
      }
    } else {
      walk(a, s, d, st, d.path, next, lane);
      st.sum = d.sum[st.cur];
      st.top = d.top[st.cur];
    }
    if (lane == 0) *out = st;
  }
  __syncthreads();
}

// What a beginning leaves: the kept rows, and, where the walk goes on in another launch, the drafts.
__device__ __forceinline__ void write_walk(const Args& a, int b, const Seq& s, const Drafts& d, const State& st, int next, bool on, int tid, int threads) {
  for (int i = tid; i < a.max_new; i += threads) a.keep[static_cast<int64_t>(b) * a.max_new + i] = i < st.count ? d.path[i] : -1;
  for (int i = tid; on && i < s.n; i += threads) {
    a.prob[s.off + i] = d.prob[i];
    a.share[s.off + i] = d.share[i];
    a.above[s.off + i] = d.above[i];
    a.row_sum[s.off + i] = d.sum[i];
    a.row_top[s.off + i] = d.top[i];
  }
  if (tid == 0 && next != kOpen) a.next[b] = next;
}

__global__ void __launch_bounds__(1024) walk_kernel(Args a, int most) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  __shared__ State st;
  __shared__ int next;
  const Drafts d(lds, most);
  const int b = blockIdx.x, tid = threadIdx.x;
  bool ok;
  const Seq s = sequence(a, b, ok);
  if (!ok && tid == 0) report(a, MOE_ERR_SLOT);
  begin(a, b, s, d, &st, &next, tid, blockDim.x);
  write_walk(a, b, s, d, st, next, st.need != kDone, tid, blockDim.x);
  if (tid == 0) {
    a.n_keep[b] = st.count;
    a.state[b] = st;
  }
}

// What one row's pass sums up, and the last one draws from.
struct Row {
  int64_t row;
  float top;
  double sum, heat, c;
};

struct Taken {   // tokens that were refused, in LDS
  int* n;
  int* token;
};

// 2^y for y <= 0, by its Taylor series in ln2 (y - rint(y)) up to the 11th power: off by 9e-15 of
// itself at most, and a rounding of 2^-53 or two.  The library's exp takes about twice the
// instructions, and a pass one a token: calls of 64 chains of 7 take 30.0 us with it, 27.7 with this; 16 trees of 31 85.0 and 80.7.
__device__ __forceinline__ double power(double y) {
  constexpr double kTerms[12] = {1.0, 0.6931471805599453, 0.24022650695910072, 0.05550410866482158, 0.009618129107628477, 0.0013333558146428443, 0.0001540353039338161, 1.5252733804059841e-05, 1.321548679014431e-06, 1.01780860092397e-07, 7.054911620801123e-09, 4.4455382718708116e-10};   // (ln 2)^k / k!
  y = fmax(y, -1100.);   // 0, of -infinity too
  const double n = __builtin_rint(y), f = y - n;
  double sum = kTerms[11];
#pragma unroll
  for (int k = 10; k >= 0; k--) sum = __fma_rn(sum, f, kTerms[k]);
  return __builtin_ldexp(sum, static_cast<int>(n));
}

// a thread's tokens' parts, from `at` on
template <int EACH>
__device__ __forceinline__ void parts_of(const Args& a, const Row& r, const Taken& out, int at, double (&v)[EACH]) {
  float x[EACH], w[EACH];
  load_some(a.type, a.logits, r.row * a.ld + at, a.vocab - at, -INFINITY, x);
  if (r.c > 0.) load_some(a.draft_type, a.draft, r.row * a.ld_draft + at, a.vocab - at, 0.f, w);
  const double rate = 1.4426950408889634 / r.heat;
#pragma unroll
  for (int e = 0; e < EACH; e++) v[e] = power((static_cast<double>(x[e]) - r.top) * rate);
  if (r.c > 0.) {
    const double scale = 1. / r.sum;
#pragma unroll
    for (int e = 0; e < EACH; e++) v[e] = fmax(v[e] * scale - r.c * static_cast<double>(w[e]), 0.);
  }
  for (int k = 0; !a.draft && k < *out.n; k++) {
    const int e0 = out.token[k] - at;
#pragma unroll
    for (int e = 0; e < EACH; e++) v[e] = e == e0 ? 0. : v[e];
  }
}

// inclusive sum over the threads before and at this one; `all` the sum of all
__device__ __forceinline__ double scan(double v, double* lds, int tid, double& all) {
  const int lane = tid % kWave, wave = tid / kWave;
  for (int w = 1; w < kWave; w <<= 1) {
    const double t = __shfl_up(v, w);
    v += lane >= w ? t : 0.;
  }
  __syncthreads();
  if (lane == kWave - 1) lds[wave] = v;
  __syncthreads();
  double before = 0.;
  all = 0.;
  for (int w = 0; w < kWaves; w++) {
    if (w < wave) before += lds[w];
    all += lds[w];
  }
  return before + v;
}

// Of the threads that have something, the first whose inclusive sum passes the aim, or the last
__device__ __forceinline__ int first_past(double mine, double up, double aim, int* lds, int tid) {
  const int wave = tid / kWave;
  const uint64_t past = __ballot(mine > 0. && up > aim), some = __ballot(mine > 0.);
  __syncthreads();
  if (tid % kWave == 0) {
    lds[2 * wave] = past ? wave * kWave + __builtin_ctzll(past) : -1;
    lds[2 * wave + 1] = some ? wave * kWave + 63 - __builtin_clzll(some) : -1;
  }
  __syncthreads();
  int at = 0;
  for (int w = 0; w < kWaves; w++)
    if (lds[2 * w + 1] >= 0) at = lds[2 * w + 1];
  for (int w = kWaves - 1; w >= 0; w--)
    if (lds[2 * w] >= 0) at = lds[2 * w];
  return at;
}

// Sums that one workgroup of a launch writes and another reads.  An exchange has been performed where
// the whole device sees it once its old value is back, which the wait is for.  (The language orders two relaxed
// operations on different places by a release alone; that the wait is in the code is tested.)
__device__ __forceinline__ void put_total(double* p, double v) {
  auto* at = reinterpret_cast<unsigned long long*>(p);
  const unsigned long long old = __hip_atomic_exchange(at, __builtin_bit_cast(unsigned long long, v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  asm volatile("s_waitcnt vmcnt(0)" : : "v"(old) : "memory");
}
__device__ __forceinline__ double read_total(const double* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// FIRST: begins the walk.
// A chain of latencies bounds it.  64 chains of 7 17.2 us, of which the beginning (lengths, drafts, their
// logits and probabilities, the walk) takes 5.6, the chunk's sum 2.7, handing it over 1.1, adding up 1.1, the draw 2.7;
// a pass of 16 trees' sequences 8.4.
template <int EACH, bool FIRST>
__global__ void __launch_bounds__(kThreads) pass_kernel(Args a, int most, int last) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  __shared__ int n_taken, next;
  const Drafts d(lds, most);
  const Taken taken{&n_taken, d.taken};
  __shared__ double parts[kWaves], carry;
  __shared__ int marks[2 * kWaves], chosen;
  __shared__ State shared;
  const int chunk = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid % kWave;
  State st;
  Seq s;
  bool ok;
  if constexpr (FIRST) {      // every workgroup of the sequence the same
    s = sequence(a, b, ok);
    if (!ok && tid == 0) report(a, MOE_ERR_SLOT);
    begin(a, b, s, d, &shared, &next, tid, kThreads);
    st = shared;
    if (st.need == kDone) {
      if (chunk == 0) write_walk(a, b, s, d, st, next, false, tid, kThreads);
      if (chunk == 0 && tid == 0) {
        a.n_keep[b] = st.count;
        a.state[b] = st;
      }
      return;
    }
  } else {
    st = a.state[b];
    if (st.need == kDone) return;
    s = sequence(a, b, ok);
    if (tid == 0) next = kOpen;
  }
  Row r;
  r.heat = heat_of(a, b);
  // what to sum next: sets r, and the tokens that are taken out of cur's row
  auto aim_at = [&]() {
    r.row = s.off + st.cur;
    r.top = st.top;
    r.sum = st.sum;
    r.c = a.draft ? st.need == kRefusal ? st.c + st.s : st.c : 0.;
    if (a.draft) return;
    __syncthreads();
    if (tid == 0) n_taken = 0;
    __syncthreads();
    if (st.s > 0.)
      for (int j = st.cur + 1 + tid; j < s.n; j += kThreads)
        if ((FIRST ? d.above[j] : a.above[s.off + j]) == st.cur) taken.token[atomicAdd(&n_taken, 1)] = a.tokens[s.off + j];
    __syncthreads();
  };
  auto chunk_sum = [&](int c) {
    double v[EACH], t = 0.;
    parts_of(a, r, taken, c * (kThreads * EACH) + tid * EACH, v);
#pragma unroll
    for (int e = 0; e < EACH; e++) t += v[e];
    t = wave_sum64(t);
    __syncthreads();
    if (lane == 0) parts[tid / kWave] = t;
    __syncthreads();
    return ((parts[0] + parts[1]) + parts[2]) + parts[3];
  };
  double* total = a.total + static_cast<int64_t>(b) * a.chunks;
  aim_at();
  const double mine = chunk_sum(chunk);
  if (tid == 0) {
    put_total(&total[chunk], mine);
    // That sum is all that workgroups of one launch hand over, so the count may go up once it is there.
    // (A release at device scope writes the whole L2 back, for each workgroup: 64 sequences by 32
    // chunks 46 us that way, 24 this way.)
    chosen = __hip_atomic_fetch_add(&a.arrived[static_cast<int64_t>(b) * kApart], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
  }
  __syncthreads();
  if (!chosen) return;
  // the last workgroup of the sequence: add up, and walk on
  if (tid == 0) a.arrived[static_cast<int64_t>(b) * kApart] = 0;
  const int each = (a.chunks + kThreads - 1) / kThreads;   // chunks of a thread, side by side
  bool loaded = FIRST;
  int* path = FIRST ? d.path : a.keep + static_cast<int64_t>(b) * a.max_new;
  for (bool summed = true;;) {
    if (!summed) {   // alone, a chunk to a wave
      aim_at();
      for (int c = tid / kWave; c < a.chunks; c += kWaves) {
        double t = 0.;
#pragma unroll 1
        for (int i = 0; i < kWaves; i++) {
          double v[EACH];
          parts_of(a, r, taken, c * (kThreads * EACH) + (i * kWave + lane) * EACH, v);
#pragma unroll
          for (int e = 0; e < EACH; e++) t += v[e];
        }
        t = wave_sum64(t);
        if (lane == 0) put_total(&total[c], t);
      }
      __syncthreads();
    }
    double have = 0., all;
    for (int c = tid * each; c < min((tid + 1) * each, a.chunks); c++) have += read_total(&total[c]);
    const double up = scan(have, parts, tid, all);
    const int need = st.need;
    bool draw = need == kDraw;
    if (need == kRefusal && !st.more && all > 0.) {    // the end: these very sums are drawn from
      st.c = r.c;
      st.s = all;
      draw = true;
    } else if (need == kRefusal) {
      const int row = st.cur;
      if (!loaded) {
        for (int i = tid; i < s.n; i += kThreads) {
          d.prob[i] = a.prob[s.off + i];
          d.share[i] = a.share[s.off + i];
          d.u[i] = a.u[s.off + i];
          d.above[i] = a.above[s.off + i];
          d.token[i] = a.tokens[s.off + i];
          d.sum[i] = a.row_sum[s.off + i];
          d.top[i] = a.row_top[s.off + i];
        }
        loaded = true;
      }
      if (all > 0.) {    // nothing left: as if it had not been refused
        st.c = r.c;
        st.s = all;
      }
      __syncthreads();
      if (tid < kWave) {
        walk(a, s, d, st, path, &next, lane);
        if (lane == 0) {
          shared = st;
          shared.sum = d.sum[st.cur];
          shared.top = d.top[st.cur];
        }
      }
      __syncthreads();
      st = shared;
      __syncthreads();
      draw = st.need == kDraw && st.cur == row && all > 0.;
    } else if (!(all > 0.) && (a.draft ? st.c > 0. : n_taken > 0)) {   // nothing left in 64 bits: the whole row
      st.c = 0.;
      st.s = -1.;
      draw = false;
    }
    if (draw) {
      const double goal = static_cast<double>(clamped(a.u_next[b])) * all;
      const int t = first_past(have, up, goal, marks, tid);
      if (tid == t) {    // the chunk among this thread's
        double before = up - have;
        int at = t * each;
        carry = before;
        for (int c = t * each; each > 1 && c < min((t + 1) * each, a.chunks); c++) {
          const double part = read_total(&total[c]);
          if (part > 0.) {
            at = c;
            carry = before;
          }
          before += part;
          if (part > 0. && before > goal) break;
        }
        chosen = at;
      }
      __syncthreads();
      const int at = chosen * (kThreads * EACH) + tid * EACH;
      const double before = carry;
      double v[EACH], have2 = 0., all2;
      parts_of(a, r, taken, at, v);
#pragma unroll
      for (int e = 0; e < EACH; e++) have2 += v[e];
      const double up2 = before + scan(have2, parts, tid, all2);
      if (tid == first_past(have2, up2, goal, marks, tid)) {
        double sum = up2 - have2;
        int x = 0;
        bool done = false;
#pragma unroll
        for (int e = 0; e < EACH; e++) {
          if (!done && v[e] > 0.) x = e;
          sum += v[e];
          done = done || (v[e] > 0. && sum > goal);
        }
        a.next[b] = at + x;
      }
      st.need = kDone;
    }
    if (st.need == kDone || !last) break;
    summed = false;
  }
  __syncthreads();
  if (FIRST) write_walk(a, b, s, d, st, next, st.need != kDone, tid, kThreads);
  else if (tid == 0 && next != kOpen) a.next[b] = next;
  if (tid == 0) {
    a.n_keep[b] = st.count;
    a.state[b] = st;
  }
}

// Statistics of a row by blocks of 16 or, where there are enough of them to fill the card twice, 32
// tokens a thread.
int each_of(int64_t n_tokens, int64_t vocab) { return n_tokens * cdiv(vocab, 16 * kThreads) > 2048 ? 32 : 16; }

// Tokens of the vocabulary for a thread of a pass: as few (4 to 16, each an exponential in 64
// bits) as take no more than 1024 workgroups, whose counts at the end would wait for each other.
int pass_each_of(int64_t n_seqs, int64_t vocab) {
  int each = 4;
  while (each < 16 && n_seqs * cdiv(vocab, each * kThreads) > 1024) each *= 2;
  return each;
}

struct Layout {
  int64_t blocks, chunks;
  size_t sum, total, row_sum, prob, state, top, row_top, share, arg, above, arrived, bytes;
};
Layout layout_of(int64_t n_seqs, int64_t n_tokens, int64_t vocab) {
  Layout l;
  l.blocks = cdiv(vocab, each_of(n_tokens, vocab) * kThreads);
  l.chunks = cdiv(vocab, pass_each_of(n_seqs, vocab) * kThreads);
  size_t at = 0;
  auto put = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 15) / 16 * 16;
    return here;
  };
  l.sum = put(8 * n_tokens * l.blocks);
  l.total = put(8 * n_seqs * l.chunks);
  l.row_sum = put(8 * n_tokens);
  l.prob = put(8 * n_tokens);
  l.state = put(sizeof(State) * n_seqs);
  l.top = put(4 * n_tokens * l.blocks);
  l.row_top = put(4 * n_tokens);
  l.share = put(4 * n_tokens);
  l.arg = put(4 * n_tokens * l.blocks);
  l.above = put(4 * n_tokens);
  l.arrived = put(4 * n_seqs * kApart);
  l.bytes = at;
  return l;
}

template <int TYPE>
void launch_stats(bool wide, int most, hipStream_t s, const Args& a) {
  const dim3 grid(a.blocks, most, a.n_seqs), block(kThreads);
  if (wide) hipLaunchKernelGGL((stats_kernel<TYPE, 32>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((stats_kernel<TYPE, 16>), grid, block, 0, s, a);
}

template <int EACH>
void launch_pass(bool first, dim3 grid, int bytes, hipStream_t s, const Args& a, int most, int last) {
  if (first) hipLaunchKernelGGL((pass_kernel<EACH, true>), grid, dim3(kThreads), bytes, s, a, most, last);
  else hipLaunchKernelGGL((pass_kernel<EACH, false>), grid, dim3(kThreads), bytes, s, a, most, last);
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
  if (!new_off || !n_keep || !next || (max_new > 0 && !keep) || (u && !u_next)) return MOE_ERR_ARG;
  if (n_tokens > 0 && (!logits || !tokens || !u != !u_next)) return MOE_ERR_ARG;
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
  Args a;
  a.logits = logits;
  a.draft = draft;
  a.tokens = tokens;
  a.parents = parents;
  a.off = new_off;
  a.temperature = temperature;
  a.u = u;
  a.u_next = u_next;
  a.keep = keep;
  a.n_keep = n_keep;
  a.next = next;
  a.status = status;
  a.sum = static_cast<double*>(part(l.sum));
  a.total = static_cast<double*>(part(l.total));
  a.row_sum = static_cast<double*>(part(l.row_sum));
  a.prob = static_cast<double*>(part(l.prob));
  a.top = static_cast<float*>(part(l.top));
  a.row_top = static_cast<float*>(part(l.row_top));
  a.share = static_cast<float*>(part(l.share));
  a.arg = static_cast<int32_t*>(part(l.arg));
  a.above = static_cast<int32_t*>(part(l.above));
  a.state = static_cast<State*>(part(l.state));
  a.arrived = static_cast<unsigned*>(part(l.arrived));
  a.ld = ld_logits;
  a.ld_draft = ld_draft;
  a.n_seqs = n_seqs;
  a.n_tokens = n_tokens;
  a.max_new = max_new;
  a.vocab = vocab;
  a.blocks = static_cast<int>(l.blocks);
  a.chunks = static_cast<int>(l.chunks);
  a.type = logits_type;
  a.draft_type = draft_type;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int most = std::min(max_new, n_tokens);
  if (most > 0) {
    const bool wide = each_of(n_tokens, vocab) == 32;
    if (logits_type == MOE_TYPE_FP32) launch_stats<MOE_TYPE_FP32>(wide, most, s, a);
    else if (logits_type == MOE_TYPE_BF16) launch_stats<MOE_TYPE_BF16>(wide, most, s, a);
    else launch_stats<MOE_TYPE_FP16>(wide, most, s, a);
  }
  // The first pass begins the walk where that takes each of its workgroups no more than a few loads (one
  // chain of 4 over 32000 tokens 16.0 us, with a launch for it 18.2; 64 chains of 7 27.7 and 30.7); else a launch with a lane for every
  // block of a sequence's rows, if that takes no more than a workgroup.
  const int64_t parts = static_cast<int64_t>(most) * a.blocks;
  const bool with_pass = most > 0 && u && parts <= 512;
  if (!with_pass) hipLaunchKernelGGL(walk_kernel, dim3(n_seqs), dim3(parts > kThreads ? 1024 : kThreads), most * kDraftBytes, s, a, most);
  if (most > 0 && u) {
    // A drawn tree takes a pass for each refusal of its walk.  What the launches leave is summed by one
    // workgroup (0.7 us a chunk: 88 us a refusal over 131072 tokens, so that a walk that refuses all of 64 drafts
    // below one row there takes 5.1 ms); one with nothing to do takes 2 us.  16 trees of 31 over 131072 tokens:
    // 77.6 us with 4, 80.7 with 6, or, where every walk refuses 5 times, 180 with 4, 97 with 6.
    const int passes = draft && parents ? std::min(most, a.chunks == 1 ? 1 : a.chunks <= 4 ? 3 : a.chunks <= 32 ? 4 : 6) : 1;
    const int bytes = most * kDraftBytes;
    const int each = pass_each_of(n_seqs, vocab);
    const dim3 grid(a.chunks, n_seqs);
    for (int i = 0; i < passes; i++) {
      const bool first = with_pass && i == 0;
      if (each == 4) launch_pass<4>(first, grid, bytes, s, a, most, i == passes - 1);
      else if (each == 8) launch_pass<8>(first, grid, bytes, s, a, most, i == passes - 1);
      else launch_pass<16>(first, grid, bytes, s, a, most, i == passes - 1);
    }
  }
  return launch_status(s);
}
