// The 4-bit cache: rows of e2m1 values (0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives; OCP microscaling formats) with one
// power-of-two scale (e8m0: code c stands for 2^(c - 127), 255 for "no number") for 32 components of a row.
//   pages   [n_pages, kv heads, block, head_dim / 2]    component 2i in the low half of byte i, 2i + 1 in the high half
//   scales  [n_pages, kv heads, head_dim / 32, block]   the scales of a group of components lie side by side for
//                                                       consecutive tokens, so that a lane reads those of 4 or 16 tokens at once
// The conversions are the chip's own; checked against the definition for every code, every bf16 value and nine scales.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

typedef __bf16 q4_bf16x2 __attribute__((ext_vector_type(2)));

// The scale code for a group whose largest magnitude has these fp32 bits: the largest value lands in [4, 7) (and those
// beyond 6 round to 6, off by less than 1, which is half of the step below them); from 7/4 of a power of two on the next
// power is taken, because such a value would round to 8, which there is not.  At most 2^125: then every stored value is a
// finite bf16 number.
__device__ __forceinline__ uint32_t q4_scale_code(uint32_t amax_bits) {
  if (amax_bits >= 0x7f800000u) return 255u;
  const int e = (int)((amax_bits + 0x200000u) >> 23) - 2;
  return (uint32_t)(e < 0 ? 0 : (e > 252 ? 252 : e));
}
// As the conversions want it: only the exponent's eight bits are looked at (zero means 2^-127).
__device__ __forceinline__ float q4_scale(uint32_t code) { return __builtin_bit_cast(float, code << 23); }

// byte SEL of `word`: its two values times the scale
template <int SEL>
__device__ __forceinline__ uint32_t q4_expand(uint32_t word, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, SEL));
}
// two bf16 values over the scale, to the nearest (ties to even), into byte SEL of `word`
template <int SEL>
__device__ __forceinline__ uint32_t q4_shrink(uint32_t word, uint32_t two, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(word, __builtin_bit_cast(q4_bf16x2, two), scale, SEL);
}
