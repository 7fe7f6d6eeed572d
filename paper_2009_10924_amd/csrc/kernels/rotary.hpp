// The angles of rotary positions.  A turn is formed in 64 bits (a position of 2^31 times a speed near 1 leaves 22 bits behind the
// point of an angle; float32 would lose whole turns from 2^24 on), reduced to an eighth of a turn around the nearest quarter,
// and only that is rounded to float32.
#pragma once
#include "device_utils.hpp"
#include "launch.hpp"

namespace fsk {

// the axis that pair i belongs to
__device__ __forceinline__ uint32_t rotary_axis(const fs::RotaryAngles& a, uint32_t i) {
  return (i >= a.end[0] ? 1u : 0u) + (i >= a.end[1] ? 1u : 0u) + (i >= a.end[2] ? 1u : 0u);
}

// Turns per position of pair i: base^-e / (2 pi), e = i / pairs (or the pair's place among its axis's own).
__device__ __forceinline__ double rotary_speed(const fs::RotaryAngles& a, uint32_t i, uint32_t axis) {
  uint32_t first = 0, of = a.pairs;
  if (a.restart) {
    first = axis == 0 ? 0u : axis == 1 ? a.end[0] : axis == 2 ? a.end[1] : a.end[2];
    of = (axis == 0 ? a.end[0] : axis == 1 ? a.end[1] : axis == 2 ? a.end[2] : a.end[3]) - first;
  }
  return exp2(-((double)(i - first) / (double)of) * a.log2_base) * 0.15915494309189533577;
}

// Cosine and sine of that many turns (their negative's, for the inverse).  Taylor's polynomials on [-pi/4, pi/4]: the first terms left
// out are below 2e-9 and 2e-10.
__device__ __forceinline__ void rotary_turn(double turns, bool inverse, float& c, float& s) {
  const double quarters = (turns - __builtin_rint(turns)) * 4.0, nearest = __builtin_rint(quarters);
  const float t = (float)((quarters - nearest) * 1.57079632679489661923), t2 = t * t;
  const float sn = t * __builtin_fmaf(t2, __builtin_fmaf(t2, __builtin_fmaf(t2, __builtin_fmaf(t2, 1.0f / 362880.0f, -1.0f / 5040.0f), 1.0f / 120.0f), -1.0f / 6.0f), 1.0f);
  const float cs = __builtin_fmaf(t2, __builtin_fmaf(t2, __builtin_fmaf(t2, __builtin_fmaf(t2, __builtin_fmaf(t2, -1.0f / 3628800.0f, 1.0f / 40320.0f), -1.0f / 720.0f), 1.0f / 24.0f), -0.5f), 1.0f);
  const int q = (int)nearest & 3;
  c = (q & 1) ? sn : cs;
  s = (q & 1) ? cs : sn;
  if (q == 1 || q == 2) c = -c;
  if ((q >= 2) != inverse) s = -s;
}

}  // namespace fsk
