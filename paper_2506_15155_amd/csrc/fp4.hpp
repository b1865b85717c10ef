// Rows of K and V in 4 bits, and 4-bit rows of codes and scales again.
//
// A block is FP4_BLOCK consecutive dims of one row. With a = max |x| over it, its scale s is the smallest power of two
// with a <= 6 s, so nothing of it is cut off; x / s is rounded to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (ties to the even
// code: what the conversion instructions do) with the sign of x. Held are the code, 4 bits with the lower dim of a pair in
// the lower half of a byte, and the scale's exponent + 127 in 8 bits. Exponents stay within -127 .. 125: values of
// the smallest magnitudes keep fewer bits, and 6 s is a finite float (blocks whose maximum is over 1.5 * 2^127 end at
// that). A block that holds a NaN or an infinity is NaN as a whole (scale 255, codes 0): neither has a code.
//
// Against the power of two that is common for such blocks, 2^(floor(log2 a) - 2), which cuts off what lies over 6 s: the
// rms error on normal values is 0.115 of theirs by either, the error of a block's largest value at most 1/5 and 1/4 of it.
#pragma once
#include "device.hpp"

namespace ellm {

constexpr int FP4_SCALE_NAN = 255, FP4_SCALE_MOST = 252;

typedef unsigned short __attribute__((ext_vector_type(2))) u16x2_t;

// the larger magnitude of either half: as integers, the magnitudes of bf16 values are in order, NaN behind infinity
__device__ __forceinline__ uint32_t max_magnitudes(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, a & 0x7fff7fffu), __builtin_bit_cast(u16x2_t, b & 0x7fff7fffu)));
}
// scale code of a block from the larger magnitudes of its halves
__device__ __forceinline__ uint32_t fp4_scale(uint32_t magnitudes) {
  const int32_t top = (int32_t)max(magnitudes & 0xffffu, magnitudes >> 16);
  // top = m 2^e, 6 = 1.5 * 2^2: the exponent goes up by one where m > 1.5
  const int32_t e = min(max(((top + 0x3f) >> 7) - 2, 0), FP4_SCALE_MOST);
  return top >= 0x7f80 ? FP4_SCALE_NAN : e;
}
// the conversion instructions take the power of two from the exponent of a float; exponent 0 is 2^-127, 255 is NaN
__device__ __forceinline__ float fp4_scale_float(uint32_t code) { return __uint_as_float(code << 23); }
// eight dims, two a word, as codes
__device__ __forceinline__ uint32_t fp4_codes(const uint32_t (&x)[4], uint32_t scale) {
  const float s = fp4_scale_float(scale);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, x[0]), s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, x[1]), s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, x[2]), s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, x[3]), s, 3);
  return scale == FP4_SCALE_NAN ? 0 : c;
}
// eight codes as bf16 values, exactly, two a word
__device__ __forceinline__ words4_t fp4_values(uint32_t codes, float scale) {
  return {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)),
          __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
          __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)),
          __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3))};
}
// the same as fp16 values, which have to be in its range
__device__ __forceinline__ words4_t fp4_values_f16(uint32_t codes, float scale) {
  return {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 0)),
          __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 1)),
          __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 2)),
          __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 3))};
}
typedef _Float16 __attribute__((ext_vector_type(2))) f16x2_t;
typedef _Float16 __attribute__((ext_vector_type(8))) f16x8_t;
// two floats rounded to nearest-even fp16, the first in the low half
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{a, b}), f16x2_t));
}
__device__ __forceinline__ f32x4_t mfma16_f16(words4_t a, words4_t b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
}
// the largest value of all lanes with the same lane & 3, in each of them
__device__ __forceinline__ uint32_t max_of_quarter(uint32_t v) {
  constexpr int ROW_ROR4 = 0x124, ROW_ROR8 = 0x128;
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ROW_ROR4, 0xf, 0xf, false));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ROW_ROR8, 0xf, 0xf, false));
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return max(b[0], b[1]);
}

// the larger of the value and that of lane ^ 1, of lane ^ 2
__device__ __forceinline__ uint32_t max_magnitudes_xor1(uint32_t m) {
  return max_magnitudes(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, DPP_QUAD_XOR1, 0xf, 0xf, false));
}
__device__ __forceinline__ uint32_t max_magnitudes_xor2(uint32_t m) {
  return max_magnitudes(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, DPP_QUAD_XOR2, 0xf, 0xf, false));
}

// bytes of a row's codes and of its scales
template <int D> constexpr int FP4_ROW = D / 2;
template <int D> constexpr int FP4_SCALES = D / FP4_BLOCK;
// Where things are in a chunk: the codes of all (kv head, plane, row), behind them the scales in the same order
template <int D>
__device__ __forceinline__ uint64_t fp4_scales_at(const PoolView& pv) { return (uint64_t)(2 * pv.n_kv_heads) * pv.tokens_per_chunk * FP4_ROW<D>; }

}  // namespace ellm
