// Elements of 8 and 4 bits that share a power of two by blocks of 32.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace gorio {

// A 16-bit element's value.
__device__ __forceinline__ float to_float(uint16_t bits, bool f16) {
  return f16 ? (float)__builtin_bit_cast(_Float16, bits) : __uint_as_float((uint32_t)bits << 16);
}

// The byte E + 127 of a block whose largest size is `most`: the smallest E in -127..127 with
// most <= M 2^E, M = 1.75 2^8 for e4m3 and 1.5 2^2 for e2m1, or 255 for a NaN or an inf.  It is
// most's own exponent less that of M, and one more where most's fraction is past M's.
template <bool k4>
__device__ __forceinline__ uint32_t mx_power(float most) {
  constexpr uint32_t kExponent = k4 ? 2 : 8, kFraction = k4 ? 0x400000 : 0x600000;
  const uint32_t bits = __float_as_uint(most), exponent = bits >> 23;
  if (exponent == 255) return 255;
  const uint32_t up = exponent + ((bits & 0x7FFFFF) > kFraction ? 1 : 0);
  return up > kExponent ? up - kExponent : 0;  // subnormals have the exponent of 2^-127, and are below M 2^-127
}

// 2^-E of a byte below 255, a normal number for 0..253 (254 is never made by mx_power).
__device__ __forceinline__ float mx_inverse(uint32_t power) { return __uint_as_float((254 - min(power, 253u)) << 23); }

// 2^E of any byte: 2^-127 is subnormal, and 255 gives NaN.
__device__ __forceinline__ float mx_factor(uint32_t power) {
  const uint32_t bits = power << 23;
  return __uint_as_float(power == 0 ? 0x00400000u : power == 255 ? 0x7FC00000u : bits);
}

// Eight values, no larger than the type's largest, to the nearest elements, ties to even.
__device__ __forceinline__ uint32_t to_e2m1(const float (&f)[8]) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[0], f[1], 1.f, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[2], f[3], 1.f, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[4], f[5], 1.f, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[6], f[7], 1.f, 3);
  return w;
}
__device__ __forceinline__ uint2 to_e4m3(const float (&f)[8]) {
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(f[i * 4], f[i * 4 + 1], 0, false);
    w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(f[i * 4 + 2], f[i * 4 + 3], w[i], true);
  }
  return make_uint2(w[0], w[1]);
}

// Eight elements to their values, exactly.
__device__ __forceinline__ void from_e2m1(uint32_t w, float (&f)[8]) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 1);
  const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 3);
  f[0] = a.x, f[1] = a.y, f[2] = b.x, f[3] = b.y, f[4] = c.x, f[5] = c.y, f[6] = d.x, f[7] = d.y;
}
__device__ __forceinline__ void from_e4m3(uint2 w, float (&f)[8]) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(w.x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w.x, true);
  const f32x2 c = __builtin_amdgcn_cvt_pk_f32_fp8(w.y, false), d = __builtin_amdgcn_cvt_pk_f32_fp8(w.y, true);
  f[0] = a.x, f[1] = a.y, f[2] = b.x, f[3] = b.y, f[4] = c.x, f[5] = c.y, f[6] = d.x, f[7] = d.y;
}

}  // namespace gorio
