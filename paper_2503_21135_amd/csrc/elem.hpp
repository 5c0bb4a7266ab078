// elem.hpp -- the element types of the decoder-block operators (MOE_TYPE_*):
// reading as fp32, and rounding to a type once (round to nearest even; NaN stays
// NaN, and fp16 overflow becomes infinity).
#pragma once

#include "common.hpp"

namespace moe {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

inline int type_bytes(int t) { return t == MOE_TYPE_FP32 ? 4 : 2; }
inline bool valid_type(int t) { return t == MOE_TYPE_BF16 || t == MOE_TYPE_FP16 || t == MOE_TYPE_FP32; }
inline bool valid_type16(int t) { return t == MOE_TYPE_BF16 || t == MOE_TYPE_FP16; }
inline bool aligned_to(const void* p, int bytes) {
  return (reinterpret_cast<uintptr_t>(p) & static_cast<uintptr_t>(bytes - 1)) == 0;
}

// whether [p, p + n) and [q, q + m) share a byte
inline bool overlap(const void* p, int64_t n, const void* q, int64_t m) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  return p && q && a < b + static_cast<uintptr_t>(m) && b < a + static_cast<uintptr_t>(n);
}


// Rows of a caller's array: n of them, each `bytes` long, `stride` bytes (>= bytes) apart.
struct Rows {
  const void* at;
  int64_t n, bytes, stride;
};
// Whether a row of p shares a byte with a row of q.  Rows of one may lie between those of the
// other (parts of one projection's rows).
inline bool overlap(const Rows& p, const Rows& q) {
  if (!overlap(p.at, (p.n - 1) * p.stride + p.bytes, q.at, (q.n - 1) * q.stride + q.bytes)) return false;
  const int64_t d = static_cast<const char*>(q.at) - static_cast<const char*>(p.at);
  if (p.stride == q.stride) {   // row j of q starts d + (j - i) stride behind row i of p
    const int64_t lo = 1 - p.n, hi = q.n - 1;   // of j - i; rows meet where -q.bytes < d + (j - i) stride < p.bytes
    const auto floor_div = [](int64_t x, int64_t y) { return x / y - (x % y < 0); };
    const int64_t first = floor_div(-q.bytes - d, p.stride) + 1, last = floor_div(p.bytes - d - 1, p.stride);
    return (first > lo ? first : lo) <= (last < hi ? last : hi);
  }
  for (int64_t i = 0; i < p.n; i++) {           // row j of q starts j * q.stride - x behind row i of p
    const int64_t x = i * p.stride - d, j = x < q.bytes ? 0 : (x - q.bytes) / q.stride + 1;
    if (j < q.n && j * q.stride - x < p.bytes) return true;
  }
  return false;
}

template <int TYPE> struct ElemOf;
template <> struct ElemOf<MOE_TYPE_BF16> { typedef __bf16 type; };
template <> struct ElemOf<MOE_TYPE_FP16> { typedef _Float16 type; };
template <> struct ElemOf<MOE_TYPE_FP32> { typedef float type; };
template <int TYPE> using elem_t = typename ElemOf<TYPE>::type;

// two values as one word of a 16-bit type
template <int TYPE>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  if constexpr (TYPE == MOE_TYPE_BF16) return __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(a), static_cast<__bf16>(b)});
  else return __builtin_bit_cast(uint32_t, f16x2{static_cast<_Float16>(a), static_cast<_Float16>(b)});
}

template <int TYPE>
__device__ __forceinline__ float half_lo(uint32_t w) {
  if constexpr (TYPE == MOE_TYPE_BF16) return bf16_lo(w);
  else return fp16_bits_to_f32(w & 0xFFFFu);
}
template <int TYPE>
__device__ __forceinline__ float half_hi(uint32_t w) {
  if constexpr (TYPE == MOE_TYPE_BF16) return bf16_hi(w);
  else return fp16_bits_to_f32(w >> 16);
}

// a . b + c over two values of a word each, exact products; and two ones
template <int TYPE>
__device__ __forceinline__ float dot2(uint32_t a, uint32_t b, float c) {
  if constexpr (TYPE == MOE_TYPE_BF16)
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, a), __builtin_bit_cast(bf16x2, b), c, false);
  else
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, a), __builtin_bit_cast(f16x2, b), c, false);
}
template <int TYPE> constexpr uint32_t kOnes = TYPE == MOE_TYPE_BF16 ? 0x3F803F80u : 0x3C003C00u;

// 16 x 16 x 32 matrix product of a 16-bit type
template <int TYPE>
__device__ __forceinline__ f32x4 product(const u32x4& a, const u32x4& b, const f32x4& c) {
  if constexpr (TYPE == MOE_TYPE_BF16) return mfma16(a, b, c);
  else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// reading and rounding with the type known at run time only
__device__ __forceinline__ float load_elem(const void* p, int64_t i, int type) {
  if (type == MOE_TYPE_FP32) return static_cast<const float*>(p)[i];
  if (type == MOE_TYPE_BF16) return static_cast<float>(static_cast<const __bf16*>(p)[i]);
  return static_cast<float>(static_cast<const _Float16*>(p)[i]);
}
__device__ __forceinline__ void store_elem(void* p, int64_t i, int type, float v) {
  if (type == MOE_TYPE_FP32) static_cast<float*>(p)[i] = v;
  else if (type == MOE_TYPE_BF16) static_cast<__bf16*>(p)[i] = static_cast<__bf16>(v);
  else static_cast<_Float16*>(p)[i] = static_cast<_Float16>(v);
}

// Reductions across lanes in vector registers alone (no pass through LDS).  A row is 16
// lanes; the swaps exchange odd rows of one register with even rows of the other, and
// its halves, so that of a register and its copy they leave each lane's own and its
// partner's value.
__device__ __forceinline__ float other_row(float v, float& own) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  own = __uint_as_float(r[0]);
  return __uint_as_float(r[1]);
}
__device__ __forceinline__ float other_half(float v, float& own) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  own = __uint_as_float(r[0]);
  return __uint_as_float(r[1]);
}
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xF, 0xF, true));
}

// over the four lanes of equal lane % 16, on all of them
__device__ __forceinline__ float rows_sum(float v) {
  float a;
  float b = other_row(v, a);
  v = a + b;
  b = other_half(v, a);
  return a + b;
}
__device__ __forceinline__ float rows_max(float v) {
  float a;
  float b = other_row(v, a);
  v = fmaxf(a, b);
  b = other_half(v, a);
  return fmaxf(a, b);
}
// over the wave, on every lane: quads, quads of 8, halves of a row, rows
__device__ __forceinline__ float wave_sum(float v) {
  v += dpp<0xB1>(v);    // lane ^ 1
  v += dpp<0x4E>(v);    // lane ^ 2
  v += dpp<0x141>(v);   // mirrored within 8
  v += dpp<0x140>(v);   // mirrored within 16
  return rows_sum(v);
}

}  // namespace moe
