// Device-side helpers of the 8-bit kernels: e4m3 elements, E8M0 scales.
#pragma once
#include <type_traits>

#include "hero_device.h"

typedef int i32x8_t __attribute__((ext_vector_type(8)));

constexpr uint32_t FP8_SCALE_ONE = 127;      // 2^0

// |v|, or 0 for NaN and infinities, which do not count for a block's scale
__device__ __forceinline__ float finite_size(float v) {
  const float s = __builtin_fabsf(v);
  return s < __builtin_inff() ? s : 0.f;
}

// largest of the 16 lanes that a block of 128 elements takes at 8 a lane
__device__ __forceinline__ float max_of_16_lanes(float v) {
  auto step = [](float x, auto CTRL) {
    const int y = __builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(CTRL)::value, 0xf, 0xf, true);
    return fmaxf(x, __int_as_float(y));
  };
  v = step(v, std::integral_constant<int, 0x128>{});     // row_ror: the row is rotated by 8, 4, 2, 1 lanes
  v = step(v, std::integral_constant<int, 0x124>{});
  v = step(v, std::integral_constant<int, 0x122>{});
  return step(v, std::integral_constant<int, 0x121>{});
}

// Scale byte of a block whose largest finite magnitude is `largest`: 2^(byte - 127) is the least power of two with
// largest <= 448 * 2^(byte - 127).  448 = 1.75 * 2^8, so the exponent is read off the bits: no division, no rounding.
__device__ __forceinline__ uint32_t fp8_scale_of(float largest) {
  const uint32_t u = __float_as_uint(largest);
  const int byte = (int)(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return u == 0 ? FP8_SCALE_ONE : (uint32_t)max(byte, 0);
}
// four values over their scale as e4m3, round to nearest even (beyond 464 and NaN: NaN).  The conversion takes the scale's
// exponent, all bytes from 0 (2^-127) on among them, and divides by it without rounding.
__device__ __forceinline__ uint32_t pack_fp8x4(float a, float b, float c, float d, uint32_t scale_byte) {
  typedef short i16x2_t __attribute__((ext_vector_type(2)));
  const float scale = __uint_as_float(scale_byte << 23);
  i16x2_t out = {0, 0};
  out = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(out, a, b, scale, false);
  out = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(out, c, d, scale, true);
  return __builtin_bit_cast(uint32_t, out);
}

// A value the compiler knows nothing of from here on: what follows from it is formed again where it is used, and not kept in
// registers from before.  (The scalar form has no meaning to the host's pass.)
template <typename T> __device__ __forceinline__ void forget(T& v) { asm volatile("" : "+v"(v)); }
template <typename T> __device__ __forceinline__ void forget_scalar(T& v) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" : "+s"(v));
#endif
}
