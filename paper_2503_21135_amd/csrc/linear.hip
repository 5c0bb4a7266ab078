// linear.hip -- moe_quant_linear: y[t][r] = bias[r] + sum_c s (q - z) x[t][c] over
// packed 4-bit rows, for few tokens.
//
// A code enters the products as the exact 16-bit number 16 + q (its 4 bits shifted into
// the mantissa of 16.0: one shift and one and-or for two codes), and each group's scale
// and zero point are applied to its fp32 partial sum:
//   sum_c s (q - z) x = s (P - (16 + z) X),  P = sum (16 + q) x,  X = sum x.
// The offset is 16, not a wider type's natural 128 or 1024, because what is taken off
// again costs fp32 bits: P is within a factor of 3 of the codes' own sum of magnitudes.
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
  int T, K, R, group, y_type;
};

template <int TYPE> constexpr uint32_t kSixteen = TYPE == MOE_TYPE_BF16 ? 0x41804180u : 0x4C004C00u;
template <int TYPE> constexpr uint32_t kCodeMask = TYPE == MOE_TYPE_BF16 ? 0x00780078u : 0x03C003C0u;

// The 8 codes of a word as 16 + q, in order.
template <int TYPE>
__device__ __forceinline__ u32x4 codes8(uint32_t w) {
  constexpr uint32_t m = kCodeMask<TYPE>, c = kSixteen<TYPE>;
  if constexpr (TYPE == MOE_TYPE_BF16)
    return u32x4{(w << 3 & m) | c, (w >> 1 & m) | c, (w >> 5 & m) | c, (w >> 9 & m) | c};
  else
    return u32x4{(w << 6 & m) | c, (w << 2 & m) | c, (w >> 2 & m) | c, (w >> 6 & m) | c};
}

template <int TYPE>
__device__ __forceinline__ float dot2(uint32_t a, uint32_t b, float c) {
  if constexpr (TYPE == MOE_TYPE_BF16)
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, a), __builtin_bit_cast(bf16x2, b), c, false);
  else
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, a), __builtin_bit_cast(f16x2, b), c, false);
}

template <int TYPE>
__device__ __forceinline__ f32x4 product(const u32x4& a, const u32x4& b, const f32x4& c) {
  if constexpr (TYPE == MOE_TYPE_BF16) return mfma16(a, b, c);
  else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

template <int TYPE> constexpr uint32_t kOnes = TYPE == MOE_TYPE_BF16 ? 0x3F803F80u : 0x3C003C00u;

__device__ __forceinline__ void store_y(const LinearArgs& a, int t, int r, float v) {
  if (a.bias) v += a.bias[r];
  store_elem(a.y, t * a.ld_y + r, a.y_type, v);
}

// One and two tokens: a wave takes RW rows, its lanes side by side along K, 32 codes
// each; no LDS and no barrier.  The activations' shares and their sums stay in registers
// for all rows of a step.
constexpr int kVecWaves = 4;

template <int TYPE, int T, int RW>
__global__ void __launch_bounds__(kVecWaves * kWave) linear_vec_kernel(LinearArgs a) {
  const int lane = threadIdx.x & 63;
  const int r0 = (blockIdx.x * kVecWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * RW;
  if (r0 >= a.R) return;
  float acc[RW][T];
#pragma unroll
  for (int r = 0; r < RW; r++)
#pragma unroll
    for (int t = 0; t < T; t++) acc[r][t] = 0.f;
  for (int k = 32 * lane; k < a.K; k += 32 * kWave) {
    u32x4 c[RW];
    uint32_t sz[RW];
    const int64_t g = k / a.group;
#pragma unroll
    for (int r = 0; r < RW; r++) {
      const int64_t row = min(r0 + r, a.R - 1);
      c[r] = *reinterpret_cast<const u32x4*>(a.codes + row * a.ld_codes + k / 8);
      sz[r] = a.sz[row * a.sz_row + g * a.sz_group];
    }
    u32x4 x[T][4];
    float sum[T];
#pragma unroll
    for (int t = 0; t < T; t++) {
      sum[t] = 0.f;
#pragma unroll
      for (int i = 0; i < 4; i++) x[t][i] = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.x) + t * a.ld_x + k + 8 * i);
#pragma unroll
      for (int i = 0; i < 4; i++)
#pragma unroll
        for (int j = 0; j < 4; j++) sum[t] = dot2<TYPE>(x[t][i][j], kOnes<TYPE>, sum[t]);
    }
#pragma unroll
    for (int r = 0; r < RW; r++) {
      float p[T];
#pragma unroll
      for (int t = 0; t < T; t++) p[t] = 0.f;
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const u32x4 w = codes8<TYPE>(c[r][i]);
#pragma unroll
        for (int j = 0; j < 4; j++)
#pragma unroll
          for (int t = 0; t < T; t++) p[t] = dot2<TYPE>(x[t][i][j], w[j], p[t]);
      }
      const float s = fp16_bits_to_f32(sz[r] & 0xFFFFu), z = fp16_bits_to_f32(sz[r] >> 16);
#pragma unroll
      for (int t = 0; t < T; t++) acc[r][t] = __fmaf_rn(s, __fmaf_rn(-(16.f + z), sum[t], p[t]), acc[r][t]);
    }
  }
#pragma unroll
  for (int r = 0; r < RW; r++)
#pragma unroll
    for (int t = 0; t < T; t++) {
      const float v = wave_sum(acc[r][t]);
      if (lane == 0 && r0 + r < a.R) store_y(a, t, r0 + r, v);
    }
}

// Three tokens and more: matrix tiles, D[token][row] += x[token][k] w[row][k], 16 tokens
// by 16 rows by 32 k.  A workgroup's waves split K in steps of 128 (16 bytes of codes a
// lane) and every wave holds NT token tiles by NR row tiles, so no operand is shared and
// there is no barrier before the waves' sums are joined through LDS.  A lane's four
// words are turned across the four lane groups (four half-swaps), which puts word 4m + g
// into group g: k = 32m + 8g .. + 7, the activations' own order.
constexpr int kTileWaves = 8;

__device__ __forceinline__ void turn4(u32x4& w) {
  auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
  auto b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
  auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
  auto d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
  w = u32x4{c[0], c[1], d[0], d[1]};
}

template <int TYPE, int GROUP, int NT, int NR>
__global__ void __launch_bounds__(kTileWaves * kWave) linear_tile_kernel(LinearArgs a) {
  constexpr int G = 128 / GROUP;   // groups of a step
  __shared__ float part[kTileWaves][NT * 16][NR * 16 + 1];
  const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r0 = blockIdx.x * NR * 16, t0 = blockIdx.y * 64;
  const int steps = (a.K + 127) / 128;
  const uint16_t* xp[NT];
#pragma unroll
  for (int n = 0; n < NT; n++)
    xp[n] = static_cast<const uint16_t*>(a.x) + static_cast<int64_t>(min(t0 + 16 * n + col, a.T - 1)) * a.ld_x + 8 * grp;
  const uint32_t *cp[NR], *sp[NR];
#pragma unroll
  for (int n = 0; n < NR; n++) {
    const int64_t row = min(r0 + 16 * n + col, a.R - 1);
    cp[n] = a.codes + row * a.ld_codes + 4 * grp;
    sp[n] = a.sz + row * a.sz_row;
  }
  f32x4 acc[NR][NT];
#pragma unroll
  for (int n = 0; n < NR; n++)
#pragma unroll
    for (int t = 0; t < NT; t++) acc[n][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  const u32x4 ones = u32x4{kOnes<TYPE>, kOnes<TYPE>, kOnes<TYPE>, kOnes<TYPE>};

  u32x4 code[NR];
  uint32_t sz[NR][G];
  auto load = [&](int st) {
#pragma unroll
    for (int n = 0; n < NR; n++) {
      // the last step of a K that is an odd number of 64s has half its words
      code[n] = 128 * st + 32 * grp < a.K ? *reinterpret_cast<const u32x4*>(cp[n] + 16 * st) : u32x4{0, 0, 0, 0};
#pragma unroll
      for (int g = 0; g < G; g++) sz[n][g] = sp[n][min(st * G + g, a.K / GROUP - 1) * a.sz_group];
    }
  };
  if (wave < steps) load(wave);
  for (int st = wave; st < steps; st += kTileWaves) {
    u32x4 now[NR];
    uint32_t szn[NR][G];
#pragma unroll
    for (int n = 0; n < NR; n++) {
      now[n] = code[n];
#pragma unroll
      for (int g = 0; g < G; g++) szn[n][g] = sz[n][g];
    }
    u32x4 x[NT][4];
#pragma unroll
    for (int t = 0; t < NT; t++)
#pragma unroll
      for (int m = 0; m < 4; m++)
        x[t][m] = 128 * st + 32 * m < a.K ? *reinterpret_cast<const u32x4*>(xp[t] + 128 * st + 32 * m) : u32x4{0, 0, 0, 0};
    if (st + kTileWaves < steps) load(st + kTileWaves);
#pragma unroll
    for (int n = 0; n < NR; n++) turn4(now[n]);
#pragma unroll
    for (int g = 0; g < G; g++) {
      constexpr int M = 4 / G;
      f32x4 sum[NT];
#pragma unroll
      for (int t = 0; t < NT; t++) {
        sum[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int m = 0; m < M; m++) sum[t] = product<TYPE>(x[t][g * M + m], ones, sum[t]);
      }
#pragma unroll
      for (int n = 0; n < NR; n++) {
        f32x4 p[NT];
#pragma unroll
        for (int t = 0; t < NT; t++) p[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int m = 0; m < M; m++) {
          const u32x4 w = codes8<TYPE>(now[n][g * M + m]);
#pragma unroll
          for (int t = 0; t < NT; t++) p[t] = product<TYPE>(x[t][g * M + m], w, p[t]);
        }
        const float s = fp16_bits_to_f32(szn[n][g] & 0xFFFFu), z = -(16.f + fp16_bits_to_f32(szn[n][g] >> 16));
#pragma unroll
        for (int t = 0; t < NT; t++)
#pragma unroll
          for (int i = 0; i < 4; i++) acc[n][t][i] = __fmaf_rn(s, __fmaf_rn(z, sum[t][i], p[t][i]), acc[n][t][i]);
      }
    }
  }
#pragma unroll
  for (int n = 0; n < NR; n++)
#pragma unroll
    for (int t = 0; t < NT; t++)
#pragma unroll
      for (int i = 0; i < 4; i++) part[wave][16 * t + 4 * grp + i][16 * n + col] = acc[n][t][i];
  __syncthreads();
  for (int i = threadIdx.x; i < NT * 16 * NR * 16; i += kTileWaves * kWave) {
    const int r = i % (NR * 16), t = i / (NR * 16);
    if (r0 + r >= a.R || t0 + t >= a.T) continue;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kTileWaves; w++) v += part[w][t][r];
    store_y(a, t0 + t, r0 + r, v);
  }
}

template <int TYPE, int T>
void launch_vec(const LinearArgs& a, hipStream_t s) {
  const auto grid = [&](int rw) { return dim3(static_cast<unsigned>(cdiv(a.R, kVecWaves * rw))); };
  if (a.R <= 8192) hipLaunchKernelGGL((linear_vec_kernel<TYPE, T, 2>), grid(2), dim3(kVecWaves * kWave), 0, s, a);
  else hipLaunchKernelGGL((linear_vec_kernel<TYPE, T, 4>), grid(4), dim3(kVecWaves * kWave), 0, s, a);
}

template <int TYPE, int GROUP, int NT>
void launch_tile(const LinearArgs& a, hipStream_t s) {
  const auto grid = [&](int nr) { return dim3(static_cast<unsigned>(cdiv(a.R, 16 * nr)), static_cast<unsigned>(cdiv(a.T, 64))); };
  if (NT == 1 || a.R < 2048) hipLaunchKernelGGL((linear_tile_kernel<TYPE, GROUP, NT, 1>), grid(1), dim3(kTileWaves * kWave), 0, s, a);
  else hipLaunchKernelGGL((linear_tile_kernel<TYPE, GROUP, NT, 2>), grid(2), dim3(kTileWaves * kWave), 0, s, a);
}

template <int TYPE, int GROUP>
void launch_tiles(const LinearArgs& a, hipStream_t s) {
  switch (a.T > 48 ? 4 : (a.T + 15) / 16) {
    case 1: launch_tile<TYPE, GROUP, 1>(a, s); break;
    case 2: launch_tile<TYPE, GROUP, 2>(a, s); break;
    case 3: launch_tile<TYPE, GROUP, 3>(a, s); break;
    default: launch_tile<TYPE, GROUP, 4>(a, s); break;
  }
}

template <int TYPE>
void launch_linear(const LinearArgs& a, hipStream_t s) {
  if (a.T == 1) launch_vec<TYPE, 1>(a, s);
  else if (a.T == 2) launch_vec<TYPE, 2>(a, s);
  else if (a.group == 64) launch_tiles<TYPE, 64>(a, s);
  else launch_tiles<TYPE, 128>(a, s);
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
  if (T < 0 || R < 0 || K <= 0 || K > INT32_MAX - 4096 || (group != 64 && group != 128) || K % group) return MOE_ERR_ARG;
  if (T > 64 * 65535 || R > INT32_MAX - 4096) return MOE_ERR_ARG;
  if (!valid_type16(x_type) || (y_type != x_type && y_type != MOE_TYPE_FP32)) return MOE_ERR_ARG;
  if (T == 0 || R == 0) return MOE_OK;
  if (!x || !codes || !sz || !y) return MOE_ERR_ARG;
  if (ld_x < K || ld_y < R || ld_codes < K / 8 || sz_row_stride < 1 || sz_group_stride < 1) return MOE_ERR_ARG;
  if (!aligned16(x) || !aligned16(codes) || ld_x % 8 || ld_codes % 4) return MOE_ERR_ALIGN;
  if (!aligned_to(sz, 4) || !aligned_to(bias, 4) || !aligned_to(y, type_bytes(y_type))) return MOE_ERR_ALIGN;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const LinearArgs a{x, codes, sz, bias, y, ld_x, ld_codes, sz_row_stride, sz_group_stride, ld_y, T, K, R, group, y_type};
  if (x_type == MOE_TYPE_BF16) launch_linear<MOE_TYPE_BF16>(a, s);
  else launch_linear<MOE_TYPE_FP16>(a, s);
  return launch_status(s);
}
