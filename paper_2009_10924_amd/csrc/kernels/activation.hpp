// The activations of the 8-bit checkpoints and of group normalisation, and division by a block's scale.
#pragma once
#include "device_utils.hpp"
#include "launch.hpp"

namespace fsk {

template <int ACT> __device__ __forceinline__ float activate(float z) {
  if constexpr (ACT == fs::ACT_GELU) return gelu_fwd(z);
  else if constexpr (ACT == fs::ACT_SILU) return z * fast_sigmoid(z);
  else return z;
}
template <int ACT> __device__ __forceinline__ float activation_slope(float z) {
  if constexpr (ACT == fs::ACT_GELU) {
    // s + z s (1 - s) d(2u)/dz with s = 1 / (1 + exp(-2u)), u = c z (1 + a z^2): 17 operations, a transcendental one counted as 4
    constexpr float c = 0.7978845608028654f, a = 0.044715f, k = -2.0f * c * kLog2e;
    const float z2 = fminf(z * z, 1e20f);   // (s is 0 or 1 long before: what it is multiplied with then has to be finite)
    const float s = fast_rcp(1.0f + __builtin_amdgcn_exp2f(z * __builtin_fmaf(k * a, z2, k)));
    const float y = z * s;
    return __builtin_fmaf(__builtin_fmaf(-y, s, y), __builtin_fmaf(6.0f * c * a, z2, 2.0f * c), s);
  } else if constexpr (ACT == fs::ACT_SILU) {
    const float s = fast_sigmoid(z);
    return s * __builtin_fmaf(z, 1.0f - s, 1.0f);
  } else return 1.0f;
}

// a block's scale, each step rounded by itself (as the graph's ops do, so that values on a rounding border of the 8-bit
// format fall to the side that they fall to there)
__device__ __forceinline__ float scale_of(float most, float inv_max, float tiny) {
#pragma clang fp contract(off)
  const float s0 = most * inv_max;
  return s0 + tiny;
}
// z / s for many z: a product with the refined reciprocal, corrected by its remainder, is the rounded quotient (but for
// cases that are rare among those the format's 4 bits can tell apart), at 3 operations where a division takes about 14.
// An infinite scale gives 0, and NaN where z is infinite too, as division does.
struct Divisor {
  float s, inv, back;
  __device__ __forceinline__ explicit Divisor(float scale) : s(scale) {
    const float r = fast_rcp(s);
    const bool finite = s < __builtin_inff();
    inv = finite ? __builtin_fmaf(__builtin_fmaf(-s, r, 1.0f), r, r) : r;
    back = finite ? s : 0.0f;
  }
  __device__ __forceinline__ float divide(float z) const {
    const float d = z * inv;
    return __builtin_fmaf(__builtin_fmaf(-d, back, z), inv, d);
  }
};

}  // namespace fsk
