// Rows in 8 and 4 bits: codes with a power of two for every 32 channels (not part of the ABI).  The conversions are the hardware's: they round
// to the nearest code, ties to even, and divide or multiply by the power of two on the way, exactly.
#pragma once

#include "wkv_device.h"
#include "wkv_generation.h"

namespace wkv {

enum { E4M3 = WKV_CACHE_E4M3, E2M1 = WKV_CACHE_E2M1 };
template <int FORMAT> constexpr int code_bytes(int d) { return FORMAT == E4M3 ? d : d / 2; }      // of a row

constexpr int SCALE_BIAS = 127, LEAST_SCALE = SCALE_BIAS - 100, NO_SCALE = 255;      // bytes; NO_SCALE: the group stands for NaN

// The scale byte of a group, from the bits of its largest magnitude (fp32, sign cleared; a NaN is larger than anything).  largest = 1.f * 2^(x - 127);
// it must not exceed 1.75 * 2^8 or 1.5 * 2^2 times the scale.
template <int FORMAT>
__device__ __forceinline__ int scale_byte(uint32_t largest) {
  constexpr int TOP = FORMAT == E4M3 ? 8 : 2;
  constexpr uint32_t FRACTION = FORMAT == E4M3 ? 0x600000 : 0x400000;
  const int s = (int)(largest >> 23) - TOP + ((largest & 0x7fffff) > FRACTION ? 1 : 0);
  return largest > 0x7f000000u ? NO_SCALE : max(s, LEAST_SCALE);
}
// (NO_SCALE gives infinity here, with which the conversions give NaN)
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Two neighbouring channels as codes into piece PART of `old` (halves of two bytes for e4m3, bytes for e2m1).
template <int FORMAT, int PART>
__device__ __forceinline__ uint32_t to_codes(uint32_t old, float a, float b, float scale) {
  typedef short s16x2 __attribute__((ext_vector_type(2)));
  if constexpr (FORMAT == E4M3)
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(__builtin_bit_cast(s16x2, old), a, b, scale, PART == 1));
  else
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(old, a, b, scale, PART);
}

// And back: piece PART of a word of codes as two bfloat16 (exact) or two floats.
template <int FORMAT, int PART>
__device__ __forceinline__ uint32_t bf16_pair(uint32_t codes, float scale) {
  if constexpr (FORMAT == E4M3) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, PART == 1));
  else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, PART));
}
template <int FORMAT, int PART>
__device__ __forceinline__ float2 float_pair(uint32_t codes, float scale) {
  if constexpr (FORMAT == E4M3) { const auto f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, scale, PART == 1); return make_float2(f[0], f[1]); }
  else { const auto f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, PART); return make_float2(f[0], f[1]); }
}

// Elements of a type as floats.
template <int DT>
__device__ __forceinline__ void widen(const uint4 &r, float *f) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (DT == DT_F32) f[i] = __uint_as_float(w[i]);
    else if constexpr (DT == DT_BF16) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    else {
      typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
      const f16x2 h = __builtin_bit_cast(f16x2, w[i]);
      f[2 * i] = (float)h[0]; f[2 * i + 1] = (float)h[1];
    }
  }
}

}  // namespace wkv
