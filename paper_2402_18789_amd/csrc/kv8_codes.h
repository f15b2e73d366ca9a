// e4m3 numbers (OCP: bias 7, largest 448, NaN 0x7f / 0xff, no infinities) and the page scales of the 8-bit cache.
#pragma once
#include "device_types.h"

namespace flexco {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// four codes of a word <-> four floats; to codes: to nearest, ties to even, values within 448 or NaN
__device__ inline void kv8_decode4(uint32_t w, float* v) {
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  v[0] = lo[0]; v[1] = lo[1]; v[2] = hi[0]; v[3] = hi[1];
}
__device__ inline uint32_t kv8_encode4(const float* v) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], w, true);
}
__device__ inline void kv8_decode16(const u32x4& w, float* v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) kv8_decode4(w[i], v + 4 * i);
}

__device__ inline bool kv8_finite(float v) { return (__builtin_bit_cast(uint32_t, v) & 0x7f800000u) != 0x7f800000u; }
// Finite numbers beyond this are stored as it is: the largest scale is 2^120, and above 1.9375 2^127 the nearest code times it is 2^128,
// an infinity in the activations' types (1.875 2^127 is off by less than 2^-4).
constexpr float KV8_MOST = 0x1.ep127f;
// what a cached element is stored from: x, or NaN for what is no finite number
__device__ inline float kv8_storable(float x) { return kv8_finite(x) ? fminf(fmaxf(x, -KV8_MOST), KV8_MOST) : __builtin_nanf(""); }

// The least 2^e >= 2^-117 with amax <= 448 2^e; amax finite, not negative.  amax = 1.f 2^E; 448 = 1.75 2^8, so e = E - 8, and one
// more where the fraction is above 1.75.  (Below 2^-117 a code times its scale could be a bf16 subnormal.)
constexpr int KV8_LEAST_EXP = -117;
__device__ inline float kv8_scale_for(float amax) {
  const uint32_t b = __builtin_bit_cast(uint32_t, amax);
  const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
  return __builtin_bit_cast(float, (uint32_t)(max(e, KV8_LEAST_EXP) + 127) << 23);
}

}  // namespace flexco
