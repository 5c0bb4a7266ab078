// linear.hip -- moe_quant_linear: y[t][r] = bias[r] + sum_c s (q - z) x[t][c] over
// packed 4-bit rows.
#include "elem.hpp"

namespace moe {
namespace {

struct LinearArgs {
  const void* x;
  const uint32_t* codes;
  const uint32_t* sz;
  const float* bias;
  void* y;
  int64_t ld_x, ld_codes, sz_row, sz_group, ld_y;
  int T, K, R, group, x_type, y_type;
};

// One wave per output row and token; a lane takes whole words (8 codes).
__global__ void __launch_bounds__(256) linear_kernel(LinearArgs a) {
  const int r = blockIdx.x * 4 + (threadIdx.x >> 6), t = blockIdx.y, lane = threadIdx.x & 63;
  if (r >= a.R) return;
  float acc = 0.f;
  for (int w = lane; w < a.K / 8; w += kWave) {
    const uint32_t c = a.codes[r * a.ld_codes + w];
    const uint32_t word = a.sz[r * a.sz_row + (8 * w / a.group) * a.sz_group];
    const float s = fp16_bits_to_f32(word & 0xFFFFu), z = fp16_bits_to_f32(word >> 16);
    float p = 0.f;
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const float q = static_cast<float>((c >> (4 * (i / 2) + 16 * (i % 2))) & 15u);
      p = __fmaf_rn(q - z, load_elem(a.x, t * a.ld_x + 8 * w + i, a.x_type), p);
    }
    acc = __fmaf_rn(s, p, acc);
  }
  for (int o = 32; o; o >>= 1) acc += __shfl_xor(acc, o);
  if (lane == 0) store_elem(a.y, t * a.ld_y + r, a.y_type, a.bias ? acc + a.bias[r] : acc);
}

}  // namespace
}  // namespace moe

extern "C" int moe_quant_linear(const void* x, int32_t x_type, int64_t ld_x, int32_t T, int32_t K,
                                const uint32_t* codes, int64_t ld_codes, const uint32_t* sz,
                                int64_t sz_row_stride, int64_t sz_group_stride, int32_t R,
                                int32_t bits, int32_t group, const float* bias, void* y,
                                int32_t y_type, int64_t ld_y, void* stream) {
  using namespace moe;
  if (bits != 4) return MOE_ERR_BITS;
  if (T < 0 || R < 0 || K <= 0 || (group != 64 && group != 128) || K % group) return MOE_ERR_ARG;
  if (!valid_type16(x_type) || (y_type != x_type && y_type != MOE_TYPE_FP32)) return MOE_ERR_ARG;
  if (T == 0 || R == 0) return MOE_OK;
  if (!x || !codes || !sz || !y) return MOE_ERR_ARG;
  if (ld_x < K || ld_y < R || ld_codes < K / 8 || sz_row_stride < 1 || sz_group_stride < 1) return MOE_ERR_ARG;
  if (!aligned16(x) || !aligned16(codes) || ld_x % 8 || ld_codes % 4) return MOE_ERR_ALIGN;
  if (!aligned_to(sz, 4) || !aligned_to(bias, 4) || !aligned_to(y, type_bytes(y_type))) return MOE_ERR_ALIGN;
  if (T > 65535) return MOE_ERR_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const LinearArgs a{x, codes, sz, bias, y, ld_x, ld_codes, sz_row_stride, sz_group_stride, ld_y,
                     T, K, R, group, x_type, y_type};
  hipLaunchKernelGGL(linear_kernel, dim3(static_cast<unsigned>(cdiv(R, 4)), T), dim3(256), 0, s, a);
  return launch_status(s);
}
