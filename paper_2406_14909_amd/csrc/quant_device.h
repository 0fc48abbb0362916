// Device helpers of the 8-bit paged cache: e4m3 numbers times a power of two for every 16
// rows of the pool.
#pragma once

#include "paged_device.h"

namespace moa {

typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kQuantLowest = -117, kQuantHighest = 119;    // exponents of scales: every number is a normal fp32 and bf16
constexpr float kQuantMost = 448.0f;                        // the largest e4m3 number

// Eight e4m3 numbers times a power of two in bf16, without rounding (one instruction per pair;
// checked on gfx950 for every code at ten scales from the least to the largest: only the exponent bits of the scale count).
__device__ __forceinline__ bf16x8 widen8(u32x2 x, float scale) {
#if defined(__HIP_DEVICE_COMPILE__)
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[0], scale, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[0], scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[1], scale, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[1], scale, true);
  return {a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
#else
  (void)x;
  (void)scale;
  return bf16x8{};
#endif
}

// Four fp32 numbers, at most 448 in magnitude or NaN, to e4m3, nearest, ties to even.
__device__ __forceinline__ uint32_t narrow4(float a, float b, float c, float d) {
#if defined(__HIP_DEVICE_COMPILE__)
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true));
#else
  (void)a, (void)b, (void)c, (void)d;
  return 0;
#endif
}

// Bit 7 of each byte that is no number.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t x) { return ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// 2^e for e in [-126, 127].
__device__ __forceinline__ float pow2(int e) { return __builtin_bit_cast(float, (e + 127) << 23); }

// e of a stored scale, as far as it can be one (0: nothing is stored yet).
__device__ __forceinline__ int quant_exponent_of(float scale) {
  const int e = static_cast<int>(__builtin_bit_cast(uint32_t, scale) >> 23 & 0xff) - 127;
  return min(max(e, kQuantLowest), kQuantHighest);
}

// The smallest e with amax <= 448 * 2^e = 1.75 * 2^(e + 8), amax >= 0 and finite.
__device__ __forceinline__ int quant_exponent(float amax) {
  const uint32_t bits = __builtin_bit_cast(uint32_t, amax);
  const int e = static_cast<int>(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return min(max(e, kQuantLowest), kQuantHighest);
}

}  // namespace moa
