// Device helpers of the attention over the 8-bit KV cache.
//
// Codes become matrix-core operands without rounding.  bf16 and f16 both hold
// every code of both formats.  Chunks and fp32 rows multiply in bf16; decodes of
// bf16 rows in f16, whose probabilities keep 11 bits instead of 8.  For int8
// f16's subnormals also make the conversion a byte move: u = code + 128 (one xor
// per four codes) put into the low byte of a half is u 2^-24.  The offset goes
// out at the end,
//   q . code = 2^24 q . (u 2^-24) - 128 sum(q),
// and alike for V with the sum of the probabilities.  q is scaled by a power of
// two into f16's range (its 8 bits fit; elements below 2^-28 of the row's
// largest lose bits; int8: rows beyond 2^111 become NaN), and the probabilities
// times their value scale are kept at the top of f16's range by a running
// maximum of their own, so they keep 11 bits; the row sum, which the value
// scales have no part in, is taken from the weights themselves where the scales
// lie so far apart that these products would lose weights.
#pragma once

#include "kv8.h"

namespace sarathi {

typedef unsigned int u32x4_nt __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_nt __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pk_bf16(float a, float b) {   // nearest even; low half = a
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t){a, b}, bf16x2_t));
}

// Four codes (a dword) to bf16: lo = codes 0, 1; hi = codes 2, 3.
template <bool INT8>
__device__ __forceinline__ void codes_bf16(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if constexpr (INT8) {
    lo = pk_bf16((float)(signed char)w, (float)(signed char)(w >> 8));
    hi = pk_bf16((float)(signed char)(w >> 16), (float)(signed char)(w >> 24));
  } else {
    lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
    hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true));
  }
}
template <bool INT8>
__device__ __forceinline__ bf16x8_t codes8_bf16(uint32_t a, uint32_t b) {
  u32x4 r;
  uint32_t x, y;
  codes_bf16<INT8>(a, x, y);
  r[0] = x; r[1] = y;
  codes_bf16<INT8>(b, x, y);
  r[2] = x; r[3] = y;
  return __builtin_bit_cast(bf16x8_t, r);
}

// x as NT bf16 terms of eight values each: bf16 rows are one exact term; fp32
// takes three (the remainders of the first two are exact in fp32), 24 bits.
template <int NT>
__device__ __forceinline__ void split8(const float* x, bf16x8_t* t) {
  float r[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = x[e];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      w[e] = pk_bf16(r[2 * e], r[2 * e + 1]);
      r[2 * e] -= __uint_as_float(w[e] << 16);
      r[2 * e + 1] -= __uint_as_float(w[e] & 0xffff0000u);
    }
    t[n] = __builtin_bit_cast(bf16x8_t, w);
  }
}

// Units of a row's sums.  The weights that multiply values are held as 2^u of
// themselves: u is 24, and -40 from the first tile on with a value scale beyond
// 2^60.  So sums of the largest values (scales below 2^122, codes 2^9, weights
// 2^8, 2^20 keys) stay in fp32's range, and the weights under the smallest scales
// (2^-100) out of its subnormals.  After the change, scales below 2^-60 count as
// that: 2^-120 of the largest.  bf16 rows take u into the exponent (and the row
// sum with it); fp32 rows, whose weights its rounding there would show in, into
// the value scale.
constexpr float KV8_UNIT = 24.f, KV8_UNIT_LARGE = -40.f;
constexpr float KV8_UNIT_STEP = 5.421010862427522e-20f;    // 2^-64: what o and l take at the change
// scale: the largest of a tile.  True: the unit changes before it.
__device__ __forceinline__ bool kv8_unit_change(float scale, float& u) {
  const bool change = scale > 1.152921504606847e18f && u > 0.f;
  u = change ? KV8_UNIT_LARGE : u;
  return change;
}
__device__ __forceinline__ float kv8_unit_pow2(float u) { return u > 0.f ? 16777216.f : 9.094947017729282e-13f; }
__device__ __forceinline__ float kv8_unit_floor(float u) { return u > 0.f ? 0.f : 8.673617379884035e-19f; }
// Out of these units: the factor for o and l, exact; or the row's maximum raised, where o may leave fp32's range:
// (m, l, o) stands for the same as (m + k, l 2^-k, o 2^-k).
__device__ __forceinline__ float kv8_unit_out(float u, float& m) {
  if (u > 0.f) return 5.9604644775390625e-8f;              // 2^-24
  m -= u;
  return 1.f;
}

typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pk_f16(float a, float b) {   // nearest even
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t){a, b}, f16x2_t));
}

// Four codes as pairs of halves (codes 0, 1 and 2, 3): int8 as u 2^-24, u = code + 128; e4m3 as they are.
__device__ __forceinline__ uint32_t offset_codes(uint32_t w) { return w ^ 0x80808080u; }
template <bool INT8>
__device__ __forceinline__ void codes_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if constexpr (INT8) {
    const uint32_t u = offset_codes(w);
    lo = __builtin_amdgcn_perm(u, u, 0x0c010c00);
    hi = __builtin_amdgcn_perm(u, u, 0x0c030c02);
  } else {
    lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false));
    hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true));
  }
}
template <bool INT8>
__device__ __forceinline__ f16x8_t codes8_f16(uint32_t a, uint32_t b) {
  uint32_t x, y, z, t;
  codes_f16<INT8>(a, x, y);
  codes_f16<INT8>(b, z, t);
  return __builtin_bit_cast(f16x8_t, (u32x4{x, y, z, t}));
}
// Byte b of eight keys' dwords as one operand (the keys along its eight elements).
template <bool INT8, bool F16>
__device__ __forceinline__ void transpose8(const uint32_t* v, u32x4* y) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (F16 && INT8) {
      const uint32_t w0 = offset_codes(v[2 * e]), w1 = offset_codes(v[2 * e + 1]);
#pragma unroll
      for (int b = 0; b < 4; ++b) y[b][e] = __builtin_amdgcn_perm(w1, w0, 0x0c040c00 + 0x00010001 * b);
    } else {
      uint32_t lo0, hi0, lo1, hi1;
      if constexpr (F16) {
        codes_f16<INT8>(v[2 * e], lo0, hi0);
        codes_f16<INT8>(v[2 * e + 1], lo1, hi1);
      } else {
        codes_bf16<INT8>(v[2 * e], lo0, hi0);
        codes_bf16<INT8>(v[2 * e + 1], lo1, hi1);
      }
      y[0][e] = __builtin_amdgcn_perm(lo1, lo0, 0x05040100);
      y[1][e] = __builtin_amdgcn_perm(lo1, lo0, 0x07060302);
      y[2][e] = __builtin_amdgcn_perm(hi1, hi0, 0x05040100);
      y[3][e] = __builtin_amdgcn_perm(hi1, hi0, 0x07060302);
    }
  }
}
// The power of two that brings a row of largest magnitude `top` to 2^14 .. 2^15, as an exponent (at most 2^`most`,
// which leaves the factor that takes it out of a score room in fp32).
__device__ __forceinline__ int f16_exponent(float top, int most) {
  return min(max((int)(__float_as_uint(top) >> 23) - 127, -100), most) - 14;
}
__device__ __forceinline__ float sum_f16(uint32_t pair, float c) {
  return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2_t, pair), (f16x2_t){(_Float16)1.f, (_Float16)1.f}, c, false);
}
__device__ __forceinline__ float sum_bf16(uint32_t pair, float c) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, pair),
                                         __builtin_convertvector((f32x2_t){1.f, 1.f}, bf16x2_t), c, false);
}

}  // namespace sarathi
