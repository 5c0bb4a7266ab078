// norm.hip -- moe_block_norm: the norm after a block, its gate, the scaled
// residual add and the norm before the next block, in one pass over each row:
//   a = y rsqrt(mean y^2 + eps) w_post,  v = beta r + alpha gate a,
//   h = v rsqrt(mean v^2 + eps) w_pre.
#include <algorithm>

#include "elem.hpp"

namespace moe {
namespace {

struct NormArgs {
  const void *y, *r, *gate;
  const float *w_post, *w_pre;
  void *r_out, *h;
  int64_t ld_y, ld_r, gate_row, gate_col, ld_r_out, ld_h;
  float branch, residual, eps;
  int64_t first;   // the launch's first row
  int T, d, y_type, r_type, gate_type, h_type;
};

constexpr int kNormThreads = 256;
constexpr int kChunk = 8;        // consecutive channels of a thread's load

// 16 bytes at any address: global accesses need no alignment here, so rows of odd
// lengths and offsets take the same loads as aligned ones
struct __attribute__((packed, aligned(2))) Words4 { uint32_t w[4]; };

struct Raw { uint32_t w[kChunk]; };   // a chunk as loaded: 8 words of fp32, 4 of a 16-bit type

__device__ __forceinline__ void load_chunk(const void* p, int64_t i, int type, int n, Raw& x) {
  if (n == kChunk) {
    const char* at = static_cast<const char*>(p) + i * (type == MOE_TYPE_FP32 ? 4 : 2);
    const Words4 lo = *reinterpret_cast<const Words4*>(at);
#pragma unroll
    for (int e = 0; e < 4; e++) x.w[e] = lo.w[e];
    if (type == MOE_TYPE_FP32) {
      const Words4 hi = *reinterpret_cast<const Words4*>(at + 16);
#pragma unroll
      for (int e = 0; e < 4; e++) x.w[4 + e] = hi.w[e];
    }
  } else if (type == MOE_TYPE_FP32) {
#pragma unroll
    for (int e = 0; e < kChunk; e++) x.w[e] = e < n ? static_cast<const uint32_t*>(p)[i + e] : 0u;
  } else {
#pragma unroll
    for (int e = 0; e < 4; e++) {
      x.w[e] = 2 * e < n ? static_cast<const uint16_t*>(p)[i + 2 * e] : 0u;
      if (2 * e + 1 < n) x.w[e] |= static_cast<uint32_t>(static_cast<const uint16_t*>(p)[i + 2 * e + 1]) << 16;
    }
  }
}

__device__ __forceinline__ void floats(const Raw& x, int type, float (&v)[kChunk]) {
  if (type == MOE_TYPE_FP32) {
#pragma unroll
    for (int e = 0; e < kChunk; e++) v[e] = __uint_as_float(x.w[e]);
  } else if (type == MOE_TYPE_BF16) {
#pragma unroll
    for (int e = 0; e < kChunk; e++) v[e] = e & 1 ? bf16_hi(x.w[e / 2]) : bf16_lo(x.w[e / 2]);
  } else {
#pragma unroll
    for (int e = 0; e < kChunk; e++) v[e] = fp16_bits_to_f32(e & 1 ? x.w[e / 2] >> 16 : x.w[e / 2] & 0xFFFFu);
  }
}

__device__ __forceinline__ void store_chunk(void* p, int64_t i, int type, int n, const float (&v)[kChunk]) {
  if (n < kChunk) {
#pragma unroll
    for (int e = 0; e < kChunk; e++)
      if (e < n) store_elem(p, i + e, type, v[e]);
    return;
  }
  char* at = static_cast<char*>(p) + i * (type == MOE_TYPE_FP32 ? 4 : 2);
  Words4 lo, hi;
  if (type == MOE_TYPE_FP32) {
#pragma unroll
    for (int e = 0; e < 4; e++) {
      lo.w[e] = __float_as_uint(v[e]);
      hi.w[e] = __float_as_uint(v[4 + e]);
    }
    *reinterpret_cast<Words4*>(at + 16) = hi;
  } else {
#pragma unroll
    for (int e = 0; e < 4; e++)
      lo.w[e] = type == MOE_TYPE_BF16 ? pack2<MOE_TYPE_BF16>(v[2 * e], v[2 * e + 1]) : pack2<MOE_TYPE_FP16>(v[2 * e], v[2 * e + 1]);
  }
  *reinterpret_cast<Words4*>(at) = lo;
}

// Sum over a row's threads (one wave, or the workgroup), in a fixed order, on every
// one of them.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* part) {
  v = wave_sum(v);
  if constexpr (TPR == kWave) return v;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  float sum = 0.f;
#pragma unroll
  for (int w = 0; w < TPR / kWave; w++) sum += part[w];
  return sum;
}

// TPR threads per row, NCH chunks of 8 channels per thread: the row is read once and
// stays in registers across both norms, each channel with the thread that writes it.
// Bound by HBM: 8192 rows of 2048 with every input (168 MB) take 36 us, 4.7 TB/s, the
// rate of a large copy; one row of 256 takes 2.8 us.
template <int TPR, int NCH>
__global__ void __launch_bounds__(TPR < kNormThreads ? kNormThreads : TPR) norm_rows_kernel(NormArgs a) {
  constexpr int kRows = TPR < kNormThreads ? kNormThreads / TPR : 1;   // rows of a workgroup
  __shared__ float part[TPR / kWave];
  const int64_t t = a.first + static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / TPR;
  if (t >= a.T) return;   // whole waves; never where a row is a workgroup's
  const int tid = threadIdx.x % TPR;
  Raw yr[NCH], rr[NCH];
  float v[NCH][kChunk];
  int at[NCH], n[NCH];
#pragma unroll
  for (int i = 0; i < NCH; i++) {
    at[i] = (tid + i * TPR) * kChunk;
    n[i] = min(max(a.d - at[i], 0), kChunk);
    if (a.y) load_chunk(a.y, t * a.ld_y + at[i], a.y_type, n[i], yr[i]);
  }
#pragma unroll
  for (int i = 0; i < NCH; i++) load_chunk(a.r, t * a.ld_r + at[i], a.r_type, n[i], rr[i]);
  Raw wr[NCH], gr[NCH], pr[NCH];   // weights and gate arrive while the row's sum is joined
#pragma unroll
  for (int i = 0; i < NCH; i++) {
    if (a.w_post) load_chunk(a.w_post, at[i], MOE_TYPE_FP32, n[i], wr[i]);
    if (a.gate && a.gate_col) load_chunk(a.gate, t * a.gate_row + at[i], a.gate_type, n[i], gr[i]);
    if (a.h && a.w_pre) load_chunk(a.w_pre, at[i], MOE_TYPE_FP32, n[i], pr[i]);
  }
  if (a.y) {
    float post = a.branch;
#pragma unroll
    for (int i = 0; i < NCH; i++) floats(yr[i], a.y_type, v[i]);
    if (a.w_post) {
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < NCH; i++)
#pragma unroll
        for (int e = 0; e < kChunk; e++) ss = __fmaf_rn(v[i][e], v[i][e], ss);
      post = a.branch / __builtin_sqrtf(row_sum<TPR>(ss, part) / static_cast<float>(a.d) + a.eps);
    }
    const float tok_gate = a.gate && !a.gate_col ? load_elem(a.gate, t * a.gate_row, a.gate_type) : 1.f;
#pragma unroll
    for (int i = 0; i < NCH; i++) {
      float r[kChunk], w[kChunk];
      floats(rr[i], a.r_type, r);
      if (a.w_post) {
        floats(wr[i], MOE_TYPE_FP32, w);
#pragma unroll
        for (int e = 0; e < kChunk; e++) v[i][e] *= w[e];
      }
      if (a.gate) {
        if (a.gate_col) {
          floats(gr[i], a.gate_type, w);
#pragma unroll
          for (int e = 0; e < kChunk; e++) v[i][e] *= w[e];
        } else {
#pragma unroll
          for (int e = 0; e < kChunk; e++) v[i][e] *= tok_gate;
        }
      }
#pragma unroll
      for (int e = 0; e < kChunk; e++) v[i][e] = __fmaf_rn(post, v[i][e], a.residual * r[e]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < NCH; i++) {
      floats(rr[i], a.r_type, v[i]);
#pragma unroll
      for (int e = 0; e < kChunk; e++) v[i][e] *= a.residual;
    }
  }
  if (a.r_out)
#pragma unroll
    for (int i = 0; i < NCH; i++) store_chunk(a.r_out, t * a.ld_r_out + at[i], a.r_type, n[i], v[i]);
  if (!a.h) return;
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < NCH; i++)
#pragma unroll
    for (int e = 0; e < kChunk; e++) ss = e < n[i] ? __fmaf_rn(v[i][e], v[i][e], ss) : ss;
  const float pre = 1.0f / __builtin_sqrtf(row_sum<TPR>(ss, part) / static_cast<float>(a.d) + a.eps);
#pragma unroll
  for (int i = 0; i < NCH; i++) {
    float w[kChunk];
    if (a.w_pre) floats(pr[i], MOE_TYPE_FP32, w);
#pragma unroll
    for (int e = 0; e < kChunk; e++) v[i][e] = a.w_pre ? v[i][e] * pre * w[e] : v[i][e] * pre;
    store_chunk(a.h, t * a.ld_h + at[i], a.h_type, n[i], v[i]);
  }
}

// Rows longer than a workgroup's registers hold: one workgroup per row, which reads the
// row again for each of the two norms.
__global__ void __launch_bounds__(kNormThreads) norm_long_kernel(NormArgs a) {
  __shared__ float part[kNormThreads / kWave];
  const int64_t t = a.first + blockIdx.x;
  float post = a.branch;
  if (a.y && a.w_post) {
    float ss = 0.f;
    for (int c = threadIdx.x; c < a.d; c += kNormThreads) {
      const float v = load_elem(a.y, t * a.ld_y + c, a.y_type);
      ss = __fmaf_rn(v, v, ss);
    }
    post = a.branch / __builtin_sqrtf(row_sum<kNormThreads>(ss, part) / static_cast<float>(a.d) + a.eps);
  }
  auto value = [&](int c) {
    float v = a.residual * load_elem(a.r, t * a.ld_r + c, a.r_type);
    if (a.y) {
      float b = load_elem(a.y, t * a.ld_y + c, a.y_type);
      if (a.w_post) b *= a.w_post[c];
      if (a.gate) b *= load_elem(a.gate, t * a.gate_row + c * a.gate_col, a.gate_type);
      v = __fmaf_rn(post, b, v);
    }
    return v;
  };
  float pre = 1.f;
  if (a.h) {
    float ss = 0.f;
    for (int c = threadIdx.x; c < a.d; c += kNormThreads) {
      const float v = value(c);
      ss = __fmaf_rn(v, v, ss);
    }
    pre = 1.0f / __builtin_sqrtf(row_sum<kNormThreads>(ss, part) / static_cast<float>(a.d) + a.eps);
  }
  for (int c = threadIdx.x; c < a.d; c += kNormThreads) {
    const float v = value(c);
    if (a.r_out) store_elem(a.r_out, t * a.ld_r_out + c, a.r_type, v);
    if (a.h) store_elem(a.h, t * a.ld_h + c, a.h_type, a.w_pre ? v * pre * a.w_pre[c] : v * pre);
  }
}

template <int TPR, int NCH>
void launch_rows(const NormArgs& a, hipStream_t s) {
  constexpr int threads = std::max(TPR, kNormThreads);
  hipLaunchKernelGGL((norm_rows_kernel<TPR, NCH>), dim3(static_cast<unsigned>(cdiv(a.T - a.first, threads / TPR))), dim3(threads), 0, s, a);
}

// As many threads as the row has chunks, so that each holds one: more chunks per thread
// mean fewer waves to hide the loads.  us, rows x channels, each pair taken together: 8192 x 2048 with 256 threads
// 34.9, with one wave of four chunks 44.5; 4096 x 4096 with 512 threads 37.3, with 256 of
// two chunks 37.7, 64 x 4096 4.5 and 6.3; 2048 x 8192 with 1024 threads 39.4, with 256 of
// four chunks 44.7.  Up to 1024 channels a wave of its own spares a row the barriers where
// there are rows enough: 16384 x 1024 with a wave 33, with 256 threads 49, 64 x 1024 5.7
// and 4.6.
void launch_norm(const NormArgs& a, hipStream_t s) {
  const int64_t chunks = cdiv(a.d, kChunk);
  if (chunks <= 64) launch_rows<64, 1>(a, s);
  else if (chunks <= 128 && a.T - a.first >= 1024) launch_rows<64, 2>(a, s);
  else if (chunks <= 256) launch_rows<256, 1>(a, s);
  else if (chunks <= 512) launch_rows<512, 1>(a, s);
  else if (chunks <= 1024) launch_rows<1024, 1>(a, s);
  else if (chunks <= 2048) launch_rows<1024, 2>(a, s);
  else hipLaunchKernelGGL(norm_long_kernel, dim3(static_cast<unsigned>(a.T - a.first)), dim3(kNormThreads), 0, s, a);
}

}  // namespace
}  // namespace moe

extern "C" int moe_block_norm(const void* y, int32_t y_type, int64_t ld_y, const void* r,
                              int32_t r_type, int64_t ld_r, int32_t T, int32_t d,
                              const float* w_post, const void* gate, int32_t gate_type,
                              int64_t gate_row_stride, int64_t gate_col_stride, float branch_scale,
                              float residual_scale, const float* w_pre, float eps, void* r_out,
                              int64_t ld_r_out, void* h, int32_t h_type, int64_t ld_h, void* stream) {
  using namespace moe;
  if (T < 0 || d <= 0 || d > (1 << 30) || !(eps >= 0.f)) return MOE_ERR_ARG;
  if (!valid_type(r_type) || (y && !valid_type(y_type)) || (gate && !valid_type(gate_type)) ||
      (h && !valid_type(h_type)))
    return MOE_ERR_ARG;
  if (!y && (w_post || gate)) return MOE_ERR_ARG;
  if (gate && (gate_row_stride < 0 || gate_col_stride < 0 || gate_col_stride > 1)) return MOE_ERR_ARG;
  if (T == 0) return MOE_OK;
  if (!r || (!r_out && !h)) return MOE_ERR_ARG;
  if (ld_r < d || (y && ld_y < d) || (r_out && ld_r_out < d) || (h && ld_h < d)) return MOE_ERR_ARG;
  if (!aligned_to(r, type_bytes(r_type)) || !aligned_to(r_out, type_bytes(r_type)) ||
      (y && !aligned_to(y, type_bytes(y_type))) || (gate && !aligned_to(gate, type_bytes(gate_type))) ||
      (h && !aligned_to(h, type_bytes(h_type))) || !aligned_to(w_post, 4) || !aligned_to(w_pre, 4))
    return MOE_ERR_ALIGN;
  // an output may be an input in place, element by element; any other overlap would
  // let one row's stores change another row's loads
  const auto bytes = [&](int64_t ld, int type) { return ((T - 1) * ld + d) * type_bytes(type); };
  const auto clash = [&](const void* in, int64_t ld_in, int type_in, const void* out, int64_t ld_out, int type_out) {
    if (!in || !out || !overlap(in, bytes(ld_in, type_in), out, bytes(ld_out, type_out))) return false;
    return in != out || type_in != type_out || (T > 1 && ld_in != ld_out);
  };
  const auto spoils = [&](const void* out, int64_t ld, int type) {   // an output that lies over an input
    if (clash(r, ld_r, r_type, out, ld, type) || (y && clash(y, ld_y, y_type, out, ld, type))) return true;
    if (gate && gate_col_stride ? clash(gate, gate_row_stride, gate_type, out, ld, type)
                                : overlap(gate, ((T - 1) * gate_row_stride + 1) * type_bytes(gate_type), out, bytes(ld, type)))
      return true;
    return overlap(w_post, 4 * static_cast<int64_t>(d), out, bytes(ld, type)) || overlap(w_pre, 4 * static_cast<int64_t>(d), out, bytes(ld, type));
  };
  if (spoils(r_out, ld_r_out, r_type) || spoils(h, ld_h, h_type)) return MOE_ERR_ARG;
  if (r_out && h && overlap(r_out, bytes(ld_r_out, r_type), h, bytes(ld_h, h_type))) return MOE_ERR_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);
  NormArgs a{y, r, gate, w_post, w_pre, r_out, h, ld_y, ld_r, gate_row_stride, gate_col_stride,
             ld_r_out, ld_h, branch_scale, residual_scale, eps, 0, T, d, y_type, r_type, gate_type, h_type};
  constexpr int64_t kRowsPerLaunch = 1 << 21;   // a grid holds 2^32 threads
  for (int64_t first = 0; first < T; first += kRowsPerLaunch) {
    a.first = first;
    a.T = static_cast<int>(std::min<int64_t>(T, first + kRowsPerLaunch));
    launch_norm(a, s);
  }
  return launch_status(s);
}
