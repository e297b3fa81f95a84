// The 8-bit cache: what a pool of dtype IC_DTYPE_E4M3 or IC_DTYPE_INT8 holds, and how codes become bf16 and back.
//
// A vector x[0..D) (one token's key or value of one head) is D codes and one scale byte b:
//   a = max |x|,  e = the smallest integer >= -100 with a <= top * 2^e  (top: 448 for e4m3, 127 for int8),
//   code = x / 2^e rounded to nearest even,  b = e + 127,  value = code * 2^e,
// and where that value is 2^128 or -2^128, which bf16 does not hold, the code below in magnitude: a finite vector has finite values.
// A power of two makes x / 2^e and code * 2^e exact: the code's rounding is the only one, and a value (4 or 7 significant bits) is a
// bf16 number, so a tile that is expanded into LDS, or read back, is the cache's content itself.  One byte a vector (M = 2 Hkv (D + 1)
// bytes a token); an fp32 scale would use the codes' range better by half a bit in the mean, and cost 3 % more bytes at head_dim 128.
// e >= -100 keeps every nonzero value (at least 2^-109) a normal number of bf16 and fp32.
// A vector with a NaN or an infinity: b = 255 and codes 0.  2^(255 - 127) as fp32 bits is infinity, and 0 * infinity is the NaN wanted.
//
// Block: codes [K | V][head][slot][dim], then scale bytes [head][K | V][slot] (32 contiguous bytes a head), rounded up to 128 bytes, so
// that every (K or V, head) tile starts on a line and a swap still moves whole blocks.
#pragma once

#include "ic_internal.h"

namespace ic {
namespace q8 {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) short s16x2;

constexpr int kE4m3 = IC_DTYPE_E4M3, kInt8 = IC_DTYPE_INT8;
constexpr uint32_t kNanBf16x2 = 0x7fc07fc0u;

// 2^(b - 127) for scale byte K of x; infinity for 255.  (One shift that selects its byte.)
template <int K>
__device__ __forceinline__ float scale_of(uint32_t x) {
  return __builtin_bit_cast(float, ((x >> (8 * K)) & 0xffu) << 23);
}

// Two codes of x as bf16: bytes 0 and 1 (kHigh: 2 and 3).  Exact.
template <int FMT, bool kHigh>
__device__ __forceinline__ uint32_t two_codes(uint32_t x) {
  if constexpr (FMT == kE4m3) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.0f, kHigh));
  } else {
    const float lo = (float)(int)(int8_t)(kHigh ? x >> 16 : x), hi = (float)(int)(int8_t)(kHigh ? x >> 24 : x >> 8);
    // a whole number of at most 8 bits: the upper half of the fp32 number is the bf16 number
    return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, hi), __builtin_bit_cast(uint32_t, lo), 0x07060302u);
  }
}
// The same times 2^e, given as fp32 (finite).
template <int FMT, bool kHigh>
__device__ __forceinline__ uint32_t two_values(uint32_t x, float scale) {
  if constexpr (FMT == kE4m3) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, kHigh));
  } else {
    const float lo = (float)(int)(int8_t)(kHigh ? x >> 16 : x) * scale, hi = (float)(int)(int8_t)(kHigh ? x >> 24 : x >> 8) * scale;
    return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, hi), __builtin_bit_cast(uint32_t, lo), 0x07060302u);
  }
}

}  // namespace q8
}  // namespace ic
