// Arithmetic that the kernels over a paged cache share: products in 16 bits, probabilities as sums of two 16-bit values, 8-bit values to
// 16 bits, sums and maxima over lanes.
#pragma once
#include "fm_cache_index.h"
#include "fm_common.h"

namespace fm {

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;

#define FM_CONSTANT __attribute__((address_space(4)))

template <bool F16>
__device__ __forceinline__ f32x4 mfma_keys(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else return mfma16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c);
}
// Two floats to 16 bits each.
template <bool F16>
__device__ __forceinline__ unsigned pack2(float a, float b) {
  if constexpr (F16) return __builtin_bit_cast(unsigned, f16x2{(_Float16)a, (_Float16)b});
  else return __builtin_bit_cast(unsigned, bf16x2{(__bf16)a, (__bf16)b});
}
// Probabilities enter their product as sums hi + lo of two 16-bit values: cut off and what that left, 16 bits of the
// value for bf16, 22 for f16.  Neither is negative, and neither is 0 where the probability is a normal number of 32 bits: an infinite
// value a row sees comes out as itself and not as 0 * inf.  For that each has the type's smallest value at least where the
// probability is above 0.  f16 ends at 2^-24: probabilities are taken times 2^kShift there, and below 2^-38 count as 2^-37.
template <bool F16>
constexpr float kShift = F16 ? 14.f : 0.f;
template <bool F16>
constexpr float kUnshift = F16 ? 0x1p-14f : 1.f;
// Two 16-bit values at least as large as two others, none of them negative: their order is that of their bits.
__device__ __forceinline__ unsigned at_least(unsigned x, u16x2 least) {
  return __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(u16x2, x), least));
}
template <bool F16>
__device__ __forceinline__ void split2(float a, float b, unsigned& hi, unsigned& lo) {
  const unsigned x = __builtin_bit_cast(unsigned, a), y = __builtin_bit_cast(unsigned, b);
  const unsigned upper = __builtin_amdgcn_perm(y, x, 0x07060302u);   // not 0 from 2^-133 on
  unsigned ones = 0x00010001u;
  asm("" : "+s"(ones));   // of a minimum with a known 1 the compiler makes comparisons of the halves one by one
  const u16x2 least = __builtin_elementwise_min(__builtin_bit_cast(u16x2, upper), __builtin_bit_cast(u16x2, ones));
  if constexpr (F16) {
    const auto h = __builtin_amdgcn_cvt_pkrtz(a, b);
    hi = at_least(__builtin_bit_cast(unsigned, h), least);
    unsigned rest = pack2<true>(a - (float)h[0], b - (float)h[1]);
    asm("" : "+v"(rest));   // one conversion of both: the compiler would take it apart
    lo = at_least(rest, least);
  } else {
    hi = upper;
    lo = at_least(pack2<false>(__builtin_bit_cast(float, x) - __builtin_bit_cast(float, x & 0xffff0000u),
                               __builtin_bit_cast(float, y) - __builtin_bit_cast(float, y & 0xffff0000u)), least);
  }
}
// Four e4m3 values to 16 bits each (exact in both types).
template <bool F16>
__device__ __forceinline__ u32x2 widen4(unsigned x) {
  if constexpr (F16)
    return u32x2{__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)x, 1.f, false)),
                 __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)x, 1.f, true))};
  else
    return u32x2{__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x, 1.f, false)),
                 __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x, 1.f, true))};
}
// The low or the high halves of two words.
__device__ __forceinline__ unsigned pair_of(unsigned first, unsigned second, int high) {
  return __builtin_amdgcn_perm(second, first, high ? 0x07060302u : 0x05040100u);
}
template <int CTRL>
__device__ __forceinline__ unsigned dpp_or(unsigned x) {
  return x | (unsigned)__builtin_amdgcn_update_dpp((int)x, (int)x, CTRL, 0xf, 0xf, false);
}
// Bits set in any of the 16 lanes of a DPP row.
__device__ __forceinline__ unsigned row16_or(unsigned x) { return dpp_or<0x121>(dpp_or<0x122>(dpp_or<0x124>(dpp_or<0x128>(x)))); }
// Whether a word of cached values has an infinity or NaN: an exponent (e4m3: all bits but the sign) of ones, to which one more bit
// carries into the sign's place.
template <bool F16, bool E4M3>
__device__ __forceinline__ bool odd_word(unsigned x) {
  constexpr unsigned kOnes = E4M3 ? 0x7f7f7f7fu : F16 ? 0x7c007c00u : 0x7f807f80u;
  constexpr unsigned kOne = E4M3 ? 0x01010101u : F16 ? 0x04000400u : 0x00800080u, kCarry = E4M3 ? 0x80808080u : 0x80008000u;
  return (((x & kOnes) + kOne) & kCarry) != 0;
}
// Whether any of eight 16-bit values is an infinity or NaN, and the values with 0 for those.
template <bool F16>
__device__ __forceinline__ bool odd_words(u32x4 x) {
  return odd_word<F16, false>(x[0]) | odd_word<F16, false>(x[1]) | odd_word<F16, false>(x[2]) | odd_word<F16, false>(x[3]);
}
template <bool F16>
__device__ __forceinline__ u32x4 without_odd(u32x4 x) {
  constexpr unsigned kOnes = F16 ? 0x7c00u : 0x7f80u;
#pragma unroll
  for (int w = 0; w < 4; ++w) x[w] &= ((x[w] & kOnes) == kOnes ? 0u : 0xffffu) | ((x[w] >> 16 & kOnes) == kOnes ? 0u : 0xffff0000u);
  return x;
}
// Maximum over the four lanes l, l ^ 16, l ^ 32, l ^ 48.
__device__ __forceinline__ float quad_max(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(int, x), __builtin_bit_cast(int, x), false, false);
  x = fmaxf(__builtin_bit_cast(float, (int)r[0]), __builtin_bit_cast(float, (int)r[1]));
  r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(int, x), __builtin_bit_cast(int, x), false, false);
  return fmaxf(__builtin_bit_cast(float, (int)r[0]), __builtin_bit_cast(float, (int)r[1]));
}
// Sums over the lanes up to this one, and the last lane's value (uniform).
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_add(int x) {
  return x + __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int wave_scan(int x) {
  x = dpp_add<0x111, 0xf>(x);   // from 1, 2, 4, 8 lanes back in the row of 16
  x = dpp_add<0x112, 0xf>(x);
  x = dpp_add<0x114, 0xf>(x);
  x = dpp_add<0x118, 0xf>(x);
  x = dpp_add<0x142, 0xa>(x);   // the last lane of rows 0 and 2 to the next row, then of row 1 to rows 2 and 3
  return dpp_add<0x143, 0xc>(x);
}
__device__ __forceinline__ int wave_last(int x) { return __builtin_amdgcn_readlane(x, 63); }
// Exponents are taken against this: a row that has seen nothing has no maximum.
__device__ __forceinline__ float reference(float m) { return m == -INFINITY ? 0.f : m; }

// Whether the bounds (LTS, LTE, UTS, UTE) of a key hide it from row i.
__device__ __forceinline__ bool hides(const i32x4& bound, int i) {
  return (bound[0] <= i && i < bound[1]) || (bound[2] <= i && i < bound[3]);
}

// Rows of [lo, hi) that the bounds of a key leave.
__device__ __forceinline__ int rows_left(int lo, int hi, const i32x4& bound) { return fm_rows_left(lo, hi, bound[0], bound[1], bound[2], bound[3]); }

}  // namespace fm
