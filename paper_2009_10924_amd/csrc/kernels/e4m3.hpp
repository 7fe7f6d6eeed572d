// 8-bit storage (e4m3: 1 sign, 4 exponent, 3 mantissa bits, largest 448, no infinities) <-> float32.
#pragma once
#include "device_utils.hpp"

namespace fsk {

struct e4m3_t { unsigned char bits; };   // storage tag type
constexpr float kE4m3Max = 448.0f;

// The conversion instruction turns what it cannot represent into NaN, so values are brought into range first (NaN stays NaN:
// the median of three would return one of the bounds).
__device__ __forceinline__ float e4m3_clamp(float x) {
  const float m = __builtin_amdgcn_fmed3f(x, -kE4m3Max, kE4m3Max);
  return x == x ? m : x;
}
// four values -> one word, round to nearest even
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_clamp(a), e4m3_clamp(b), 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_clamp(c), e4m3_clamp(d), w, true);
  return (uint32_t)w;
}
// the same for values of at most 448 but for their rounding (which the format's next border, 464, is far from), or NaN
__device__ __forceinline__ uint32_t pack_e4m3_in_range(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  return (uint32_t)w;
}
__device__ __forceinline__ void store1_in_range(e4m3_t* p, float v) { p->bits = (unsigned char)(__builtin_amdgcn_cvt_pk_fp8_f32(v, 0.0f, 0, false) & 0xFF); }
__device__ __forceinline__ void unpack_e4m3(uint32_t w, float& a, float& b, float& c, float& d) {
  const f32x2 lo = __builtin_bit_cast(f32x2, __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false));
  const f32x2 hi = __builtin_bit_cast(f32x2, __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true));
  a = lo.x; b = lo.y; c = hi.x; d = hi.y;
}
__device__ __forceinline__ float load1(const e4m3_t* p) {
  return __builtin_amdgcn_cvt_f32_fp8((int)p->bits, 0);
}
__device__ __forceinline__ void store1(e4m3_t* p, float v) {
  p->bits = (unsigned char)(__builtin_amdgcn_cvt_pk_fp8_f32(e4m3_clamp(v), 0.0f, 0, false) & 0xFF);
}
__device__ __forceinline__ void load_vec4(const e4m3_t* p, float (&v)[4]) {
  unpack_e4m3(*reinterpret_cast<const uint32_t*>(p), v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void load_vec(const e4m3_t* p, float (&v)[8]) {
  const u32x2 t = *reinterpret_cast<const u32x2*>(p);
  unpack_e4m3(t.x, v[0], v[1], v[2], v[3]);
  unpack_e4m3(t.y, v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store_vec4(e4m3_t* p, const float (&v)[4]) {
  *reinterpret_cast<uint32_t*>(p) = pack_e4m3(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void store_vec(e4m3_t* p, const float (&v)[8]) {
  const u32x2 t = {pack_e4m3(v[0], v[1], v[2], v[3]), pack_e4m3(v[4], v[5], v[6], v[7])};
  *reinterpret_cast<u32x2*>(p) = t;
}

}  // namespace fsk
