// The 8-bit key/value cache: conversions shared by its kernels.
//
// A page holds B tokens of every key/value head as e4m3 codes, keys
// [page][head][B][d] and values [page][head][d][B] (transposed: a lane of the
// attention's P V product then loads 16 tokens of its value dimension in one
// piece, in the operand layout of the matrix instruction). Each (page, head)
// has one power of two for its keys and one for its values, kept as the byte
// exponent + 127. The code is a floating-point number, so a scale with a
// mantissa would gain no precision; with a power of two x / scale is exact,
// the code is the one rounding (to nearest even, at most 2^-4 relative; steps
// of 2^-9 scale below 2^-6 scale), a decoded value is exact in bfloat16, and a
// block whose scale has to grow loses nothing but what falls below that step.
#pragma once

#include "sw_common.h"

namespace sw {

typedef __bf16 bf16x2q __attribute__((ext_vector_type(2)));
typedef float f32x2q __attribute__((ext_vector_type(2)));

// 2^(b - 127).
__device__ __forceinline__ float q8_scale(uint32_t b) {
  return __uint_as_float(b ? b << 23 : 0x00400000u);
}

// The smallest e in [-126, 127] with amax <= 448 * 2^e (448 = 1.75 * 2^8 is the
// largest code); amax finite, >= 0.
__device__ __forceinline__ int q8_exponent(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 135 + ((u & 0x7fffffu) > 0x600000u);
  return max(e, -126);
}

// The four codes of a word, times m (a power of two of at most 1), rounded again.
__device__ __forceinline__ uint32_t q8_rescale4(uint32_t w, float m) {
  const f32x2q a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  const f32x2q b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a[0] * m, a[1] * m, 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(b[0] * m, b[1] * m, r, true);
  return (uint32_t)r;
}

}  // namespace sw
