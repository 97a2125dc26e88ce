// The 8-bit cache's numbers on the device: e4m3 (1 sign, 4 exponent, 3 mantissa bits; largest
// 448, smallest 2^-9, NaN but no infinities) under a power of two for each slot's keys and
// values.
#pragma once

#include "spla_device.h"

namespace spla {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float float2_t __attribute__((ext_vector_type(2)));

// 8 codes times scale, a power of two, as 8 bf16 (exact: 4 significant bits).
__device__ __forceinline__ uint4 fp8_to_bf16(uint32_t lo, uint32_t hi, float scale) {
  uint4 r;
  r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false));
  r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true));
  r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false));
  r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true));
  return r;
}

// The NaN codes (magnitude 0x7F) among 4, as their top bits.
__device__ __forceinline__ uint32_t fp8_nan(uint32_t w) {
  return ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
}

// 4 fp32 times inv, a power of two, to the nearest codes (ties to even): finite magnitudes past
// 448 become 448, infinities and NaN become NaN. (The instruction's own answer to them depends on
// a mode, so they do not reach it.)
__device__ __forceinline__ uint32_t fp8_round4(const float (&x)[4], float inv) {
  uint32_t nan = 0u;
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool odd = (__float_as_uint(x[i]) & 0x7F800000u) == 0x7F800000u;
    nan |= odd ? 0x7Fu << (8 * i) : 0u;
    y[i] = odd ? 0.f : fminf(fmaxf(x[i] * inv, -448.f), 448.f);
  }
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
  return (uint32_t)w | nan;
}

// 4 codes under one power of two rewritten under another, larger by 1 / f: what is below its
// steps is rounded; NaN stays.
__device__ __forceinline__ uint32_t fp8_rescale4(uint32_t w, float f) {
  const float2_t a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  const float2_t b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  const float x[4] = {a[0], a[1], b[0], b[1]};
  return fp8_round4(x, f);
}

// 2^e from its exponent, -126 <= e <= 127, and back.
__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
__device__ __forceinline__ int exponent_of(float s) { return (int)(__float_as_uint(s) >> 23) - 127; }

// The smallest e with amax <= 448 2^e (448 = 1.75 2^8), within the range of the scales.
__device__ __forceinline__ int fp8_exponent(uint32_t amax_bits) {
  const int e = (int)(amax_bits >> 23) - 127 - 8 + ((amax_bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return min(max(e, kScale8Min), kScale8Max);
}

}  // namespace spla
