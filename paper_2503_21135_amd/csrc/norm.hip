// norm.hip -- moe_block_norm: the norm after a block, its gate, the scaled
// residual add and the norm before the next block, in one pass over each row:
//   a = y rsqrt(mean y^2 + eps) w_post,  v = beta r + alpha gate a,
//   h = v rsqrt(mean v^2 + eps) w_pre.
#include "elem.hpp"

namespace moe {
namespace {

struct NormArgs {
  const void *y, *r, *gate;
  const float *w_post, *w_pre;
  void *r_out, *h;
  int64_t ld_y, ld_r, gate_row, gate_col, ld_r_out, ld_h;
  float branch, residual, eps;
  int T, d, y_type, r_type, gate_type, h_type;
};

constexpr int kNormThreads = 256;

// Sum over the workgroup, in a fixed order, on every thread.
__device__ __forceinline__ float block_sum(float v, float* part) {
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  return (part[0] + part[1]) + (part[2] + part[3]);
}

// One workgroup per row; the row is read again for each of the two norms.
__global__ void __launch_bounds__(kNormThreads) norm_kernel(NormArgs a) {
  __shared__ float part[kNormThreads / kWave];
  const int64_t t = blockIdx.x;
  float post = 1.f;
  if (a.y && a.w_post) {
    float ss = 0.f;
    for (int c = threadIdx.x; c < a.d; c += kNormThreads) {
      const float v = load_elem(a.y, t * a.ld_y + c, a.y_type);
      ss = __fmaf_rn(v, v, ss);
    }
    post = 1.0f / __builtin_sqrtf(block_sum(ss, part) / static_cast<float>(a.d) + a.eps);
  }
  auto value = [&](int c) {
    float v = a.residual * load_elem(a.r, t * a.ld_r + c, a.r_type);
    if (a.y) {
      float b = load_elem(a.y, t * a.ld_y + c, a.y_type);
      if (a.w_post) b *= post * a.w_post[c];
      if (a.gate) b *= load_elem(a.gate, t * a.gate_row + c * a.gate_col, a.gate_type);
      v = __fmaf_rn(a.branch, b, v);
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
    pre = 1.0f / __builtin_sqrtf(block_sum(ss, part) / static_cast<float>(a.d) + a.eps);
  }
  for (int c = threadIdx.x; c < a.d; c += kNormThreads) {
    const float v = value(c);
    if (a.r_out) store_elem(a.r_out, t * a.ld_r_out + c, a.r_type, v);
    if (a.h) store_elem(a.h, t * a.ld_h + c, a.h_type, a.w_pre ? v * pre * a.w_pre[c] : v * pre);
  }
}

// whether [p, p + n) and [q, q + m) share a byte
bool overlap(const void* p, int64_t n, const void* q, int64_t m) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  return p && q && a < b + static_cast<uintptr_t>(m) && b < a + static_cast<uintptr_t>(n);
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
  if (clash(r, ld_r, r_type, r_out, ld_r_out, r_type) || clash(r, ld_r, r_type, h, ld_h, h_type) ||
      (y && (clash(y, ld_y, y_type, r_out, ld_r_out, r_type) || clash(y, ld_y, y_type, h, ld_h, h_type))))
    return MOE_ERR_ARG;
  if (r_out && h && overlap(r_out, bytes(ld_r_out, r_type), h, bytes(ld_h, h_type))) return MOE_ERR_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const NormArgs a{y, r, gate, w_post, w_pre, r_out, h, ld_y, ld_r, gate_row_stride, gate_col_stride,
                   ld_r_out, ld_h, branch_scale, residual_scale, eps, T, d, y_type, r_type, gate_type, h_type};
  hipLaunchKernelGGL(norm_kernel, dim3(static_cast<unsigned>(T)), dim3(kNormThreads), 0, s, a);
  return launch_status(s);
}
