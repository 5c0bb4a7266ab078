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

// The 8 codes of a word as 16 + q, in order.  `c` holds kSixteen in a vector register: as
// a second literal it would split the and-or in two.
template <int TYPE>
__device__ __forceinline__ u32x4 codes8(uint32_t w, uint32_t c) {
  constexpr uint32_t m = kCodeMask<TYPE>;
  if constexpr (TYPE == MOE_TYPE_BF16)
    return u32x4{(w << 3 & m) | c, (w >> 1 & m) | c, (w >> 5 & m) | c, (w >> 9 & m) | c};
  else
    return u32x4{(w << 6 & m) | c, (w << 2 & m) | c, (w >> 2 & m) | c, (w >> 6 & m) | c};
}

template <int TYPE>
__device__ __forceinline__ uint32_t sixteen() {
  uint32_t c = kSixteen<TYPE>;
  asm("" : "+v"(c));
  return c;
}

__device__ __forceinline__ void store_y(const LinearArgs& a, int t, int r, float v) {
  if (a.bias) v += a.bias[r];
  store_elem(a.y, t * a.ld_y + r, a.y_type, v);
}

// One token, and two by few rows: a wave takes RW rows, its lanes side by side along K, 32 codes
// each; no LDS and no barrier.  The activations' shares and their sums stay in registers
// for all rows of a step.  Bound by HBM where there are many rows (one token by 32000 x
// 4096, 70 MB: 15.0 us, 4.6 TB/s), else by the chain of loads (4096 x 4096: 4.4 us).
constexpr int kVecWaves = 4;

template <int TYPE, int T, int RW>
__global__ void __launch_bounds__(kVecWaves * kWave) linear_vec_kernel(LinearArgs a) {
  const int lane = threadIdx.x & 63;
  const int r0 = (blockIdx.x * kVecWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * RW;
  if (r0 >= a.R) return;
  const uint32_t sixteens = sixteen<TYPE>();
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
        const u32x4 w = codes8<TYPE>(c[r][i], sixteens);
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

// More tokens: matrix tiles, D[token][row] += x[token][k] w[row][k], 16 tokens
// by 16 rows by 32 k, K in steps of 128 (16 bytes of codes a lane).
//
// A workgroup of W waves is RW row waves, NR row tiles each, by KW = W / RW K waves, which
// take every KW-th step and are joined through LDS at the end.  The row waves of a step
// share its activations through LDS: 16 lanes read a token's 256 bytes side by side (a
// matrix operand taken straight from memory has 16 tokens side by side instead, whose
// 16-byte pieces the vector memory path serves one per cycle: 64 tokens by 32000 rows
// took 73 us that way), and the same 16 lanes form the token's sums X.  Two buffers, one
// barrier a step; the next step's activations and codes are on their way during the
// products.
//
// 64 tokens by 32000 x 4096 (78 MB, 16.8 GFLOP) take 33.1 us; the vector instructions
// (unpacking, scale and zero point, staging: 278 per wave and step beside 32 matrix
// instructions) fill about half of the issue slots, the waits around the barrier most of
// the rest.  Prefetching codes four steps ahead, activations two, or the LDS operands one
// product ahead changed nothing (37.3, 37.3 and 35.6 us against 37.2 and 35.1, on a card that had rested).
//
// A lane's four code words are turned across the four lane groups (four half-swaps),
// which puts word 4m + g into group g: k = 32m + 8g .. + 7, the activations' own order.

__device__ __forceinline__ void turn4(u32x4& w) {
  auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
  auto b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
  auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
  auto d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
  w = u32x4{c[0], c[1], d[0], d[1]};
}

template <int TYPE, int GROUP, int NT, int W, int RW, int NR>
__global__ void __launch_bounds__(W * kWave) linear_tile_kernel(LinearArgs a) {
  constexpr int G = 128 / GROUP;             // groups of a step
  constexpr int KW = W / RW, TOK = NT * 16, ROWS = RW * NR * 16;
  constexpr int NL = TOK * 16 / (RW * kWave);   // 16-byte pieces of a step that a thread stages
  struct Stage {
    u32x4 x[KW][TOK][16];      // piece c of token t at c ^ (t % 16): operand reads hit all banks
    float sum[KW][G][TOK];
  };
  union Lds {
    Stage stage[2];
    float part[KW][TOK][ROWS + 1];
  };
  __shared__ Lds lds;
  const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kw = wave / RW, rw = wave % RW, in_kw = threadIdx.x % (RW * kWave);
  const int r0 = blockIdx.x * ROWS, t0 = blockIdx.y * 64;
  const int steps = (a.K + 127) / 128, rounds = (steps + KW - 1) / KW;
  const uint32_t sixteens = sixteen<TYPE>();
  f32x4 acc[NR][NT];
#pragma unroll
  for (int n = 0; n < NR; n++)
#pragma unroll
    for (int t = 0; t < NT; t++) acc[n][t] = f32x4{0.f, 0.f, 0.f, 0.f};

  // next step's pieces; the pointers move with the steps, and what a step has past the end
  // of K is zeros among the activations and any codes
  const int pc = in_kw % 16, pt = in_kw / 16;      // this thread's piece, and its first token
  const uint16_t* xp[NL];
  const uint32_t *cp[NR], *sp[NR];
#pragma unroll
  for (int i = 0; i < NL; i++)
    xp[i] = static_cast<const uint16_t*>(a.x) + static_cast<int64_t>(min(t0 + pt + i * (RW * 4), a.T - 1)) * a.ld_x;
#pragma unroll
  for (int n = 0; n < NR; n++) {
    const int64_t row = min(r0 + (rw * NR + n) * 16 + col, a.R - 1);
    cp[n] = a.codes + row * a.ld_codes;
    sp[n] = a.sz + row * a.sz_row;
  }
  u32x4 code[NR], xs[NL];
  uint32_t sz[NR][G];
  auto load = [&](int st) {
    const int k = 128 * st + 8 * pc, kx = min(k, a.K - 8), kc = min(128 * st + 32 * grp, a.K - 32) / 8;
#pragma unroll
    for (int i = 0; i < NL; i++) xs[i] = *reinterpret_cast<const u32x4*>(xp[i] + kx);
    if (128 * (st + 1) > a.K)
#pragma unroll
      for (int i = 0; i < NL; i++) xs[i] = k < a.K ? xs[i] : u32x4{0, 0, 0, 0};
#pragma unroll
    for (int n = 0; n < NR; n++) {
      code[n] = *reinterpret_cast<const u32x4*>(cp[n] + kc);
#pragma unroll
      for (int g = 0; g < G; g++) sz[n][g] = sp[n][min(st * G + g, a.K / GROUP - 1) * a.sz_group];
    }
  };
  load(kw);
  for (int round = 0; round < rounds; round++) {
    Stage& stage = lds.stage[round & 1];
    float mine = 0.f;      // the sum that this lane writes: of its row's piece pc % (16 / G)
#pragma unroll
    for (int i = 0; i < NL; i++) {
      float v = 0.f;
#pragma unroll
      for (int j = 0; j < 4; j++) v = dot2<TYPE>(xs[i][j], kOnes<TYPE>, v);
      v += dpp<0xB1>(v);
      v += dpp<0x4E>(v);
      v += dpp<0x141>(v);
      if constexpr (G == 1) v += dpp<0x140>(v);
      mine = pc % (16 / G) == i ? v : mine;
      const int t = pt + i * (RW * 4);
      stage.x[kw][t][pc ^ (t & 15)] = xs[i];
    }
    if (pc % (16 / G) < NL) stage.sum[kw][pc * G / 16][pt + pc % (16 / G) * (RW * 4)] = mine;
    u32x4 now[NR];
    uint32_t szn[NR][G];
#pragma unroll
    for (int n = 0; n < NR; n++) {
      now[n] = code[n];
      turn4(now[n]);
#pragma unroll
      for (int g = 0; g < G; g++) szn[n][g] = sz[n][g];
    }
    __syncthreads();
    if (round + 1 < rounds) load((round + 1) * KW + kw);
#pragma unroll
    for (int g = 0; g < G; g++) {
      constexpr int M = 4 / G;
      const f32x4 zero = f32x4{0.f, 0.f, 0.f, 0.f};
      f32x4 p[NR][NT];
#pragma unroll
      for (int m = 0; m < M; m++) {
        u32x4 x[NT];
#pragma unroll
        for (int t = 0; t < NT; t++) x[t] = stage.x[kw][16 * t + col][(4 * (g * M + m) + grp) ^ col];
#pragma unroll
        for (int n = 0; n < NR; n++) {
          const u32x4 w = codes8<TYPE>(now[n][g * M + m], sixteens);
#pragma unroll
          for (int t = 0; t < NT; t++) p[n][t] = product<TYPE>(x[t], w, m ? p[n][t] : zero);
        }
      }
#pragma unroll
      for (int t = 0; t < NT; t++) {
        const f32x4 sum = *reinterpret_cast<const f32x4*>(&stage.sum[kw][g][16 * t + 4 * grp]);
#pragma unroll
        for (int n = 0; n < NR; n++) {
          const float s = fp16_bits_to_f32(szn[n][g] & 0xFFFFu), z = -(16.f + fp16_bits_to_f32(szn[n][g] >> 16));
#pragma unroll
          for (int i = 0; i < 4; i++) acc[n][t][i] = __fmaf_rn(s, __fmaf_rn(z, sum[i], p[n][t][i]), acc[n][t][i]);
        }
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int n = 0; n < NR; n++)
#pragma unroll
    for (int t = 0; t < NT; t++)
#pragma unroll
      for (int i = 0; i < 4; i++) lds.part[kw][16 * t + 4 * grp + i][(rw * NR + n) * 16 + col] = acc[n][t][i];
  __syncthreads();
  for (int i = threadIdx.x; i < TOK * ROWS; i += W * kWave) {
    const int r = i % ROWS, t = i / ROWS;
    if (r0 + r >= a.R || t0 + t >= a.T) continue;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < KW; w++) v += lds.part[w][t][r];
    store_y(a, t0 + t, r0 + r, v);
  }
}

// Two rows a wave while rows are few, four where there are many (one token, us, two and four:
// 4096 rows 4.3 and 4.7, 9000 6.6 and 7.3, 16000 9.0 and 9.4, 32000 15.0 and 15.0, 128000 71.3
// and 69.1).
template <int TYPE, int T, int RW>
void launch_vec(const LinearArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((linear_vec_kernel<TYPE, T, RW>), dim3(static_cast<unsigned>(cdiv(a.R, kVecWaves * RW))), dim3(kVecWaves * kWave),
                     0, s, a);
}

template <int TYPE, int GROUP, int NT, int W, int RW, int NR>
void launch_tile(const LinearArgs& a, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(cdiv(a.R, RW * NR * 16)), static_cast<unsigned>(cdiv(a.T, 64)));
  hipLaunchKernelGGL((linear_tile_kernel<TYPE, GROUP, NT, W, RW, NR>), grid, dim3(W * kWave), 0, s, a);
}

// Rows of a workgroup: few while there are few rows to spread over the machine, more
// when each workgroup's pass over the activations costs more than it spreads.  us, K 4096:
//   64 tokens   4096 rows: 32 a workgroup 16.5, 64 18.0, 128 29.3;  12000: 31.9, 19.5, 30.2;
//               32000: 66.5, 39.0, 35.1
//   37 tokens   6144 rows: 32 a workgroup 14.3, 64 16.1
//   16 tokens   6144 rows: 16 a workgroup 8.8, 32 9.0, 64 10.0;  32000: 32 18.5, 64 15.9, 128 17.9
//   5 tokens    4096 rows: 16 a workgroup 6.0, 32 7.4, 64 8.8
// (each line taken together, on a card that had rested; after some hundred calls the chosen
// ones take 16.0, 18.0, 32.0; 12.5; 8.2, 15.4; 5.9)
template <int TYPE, int GROUP, int NT>
void launch_tile(const LinearArgs& a, hipStream_t s) {
  if (a.R > 8192) {
    if constexpr (NT > 2) {
      if (a.R > 20480) return launch_tile<TYPE, GROUP, NT, 8, 4, 2>(a, s);
    }
    launch_tile<TYPE, GROUP, NT, 16, 4, 1>(a, s);
  } else {
    launch_tile<TYPE, GROUP, NT, 8, NT == 1 ? 1 : 2, 1>(a, s);
  }
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

// Two tokens take dot products while rows are few (us, taken together on a card that had
// rested: 4096 rows 5.6, matrix tiles 6.0; 32000 rows 20.6 and 16.2).
template <int TYPE>
void launch_linear(const LinearArgs& a, hipStream_t s) {
  if (a.T == 1 && a.R <= 8192) launch_vec<TYPE, 1, 2>(a, s);
  else if (a.T == 1) launch_vec<TYPE, 1, 4>(a, s);
  else if (a.T == 2 && a.R <= 8192) launch_vec<TYPE, 2, 2>(a, s);
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
  if (T > 64 * 65535 || R > (1 << 27)) return MOE_ERR_ARG;   // what one grid holds
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
