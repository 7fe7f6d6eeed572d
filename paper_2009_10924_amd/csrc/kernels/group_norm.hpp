// What the group normalisation kernels share: which channels and positions a thread of a workgroup has, and the sums of its
// group's values.
//
// x is [batch, positions, channels], channel = group * dim + d.  A workgroup works on a set of `set_groups` groups (`width`
// neighbouring channels) of one batch entry.  Thread t has the vector t % set_vecs of the set's channels, at positions
// t / set_vecs, + rows_at_once, + 2 rows_at_once, ...: its channels stay the same, so what is per channel is loaded once, and
// neighbouring threads read neighbouring memory.  The last vector of a set starts early where the width is no multiple of VEC;
// the channels it then shares with its neighbour have the same values in both and are deposited twice in the same place.
#pragma once
#include <type_traits>

#include "activation.hpp"
#include "kernel_arguments.hpp"
#include "vec_access.hpp"

namespace fsk {
using fs::GnShape;

struct GnLane {
  uint32_t row, vec, col;   // first position, vector within the set, its first channel within the set
  bool live;                // threads beyond rows_at_once * set_vecs have nothing
};
template <int VEC>
__device__ __forceinline__ GnLane gn_lane(const GnShape& p) {
  GnLane l;
  l.row = (threadIdx.x * p.set_vecs_m) >> 20;   // exact for 1024 threads: the factor is off by less than 2^-20 * set_vecs
  l.vec = threadIdx.x - l.row * p.set_vecs;
  l.col = min(l.vec * VEC, p.set_groups * p.dim - VEC);
  l.live = l.row < p.rows_at_once;
  return l;
}

// gamma or beta of a thread's channels, from channel `at` on: stored like x, or (wide) in float32 beside a 16-bit x.  Loaded without a
// branch, whose end would wait for these loads and all before them (2 to 3 % of calls with two launches), so the second half of
// wide ones is always loaded, of the others the first again.
template <typename T, int VEC>
struct GnParams {
  static constexpr bool kHalves = sizeof(T) < 4;
  typedef typename std::conditional<VEC == 1 && kHalves, uint16_t, typename VecIo<T, VEC>::Raw>::type Raw;
  Raw lo, hi;
  __device__ __forceinline__ static Raw one(const T* p) {
    if constexpr (VEC == 1 && kHalves) return *reinterpret_cast<const uint16_t*>(p);
    else return VecIo<T, VEC>::template load<false>(p);
  }
  __device__ __forceinline__ void load(const T* from, uint32_t at, bool wide) {
    const T* const p = from + at + (kHalves && wide ? at : 0u);
    lo = one(p);
    if constexpr (kHalves) hi = one(wide ? p + VEC : p);
  }
  __device__ __forceinline__ void widen(bool wide, float (&v)[VEC]) const {
    if constexpr (VEC == 1 && kHalves) {
      const T own = __builtin_bit_cast(T, lo);
      v[0] = wide ? __builtin_bit_cast(float, (uint32_t)lo | (uint32_t)hi << 16) : load1(&own);
    } else {
      VecIo<T, VEC>::widen(lo, v);
      if constexpr (kHalves) {
        if (wide) {
          const f32x4 a = __builtin_bit_cast(f32x4, lo), b = __builtin_bit_cast(f32x4, hi);
          const float w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
          for (int e = 0; e < VEC; ++e) v[e] = w[e];
          done(v);   // (a branch, not a choice per value)
        }
      }
    }
  }
};

// Workgroups go to the dies in turn; neighbouring sets, which share lines of memory, belong on one die and behind its cache.
__device__ __forceinline__ uint32_t gn_block(uint32_t blocks) {
  const uint32_t b = blockIdx.x;
  return (blocks & 7u) == 0 ? (b & 7u) * (blocks >> 3) + (b >> 3) : b;
}

// What a workgroup's threads have gathered, in LDS for others to add up: gn_pitch items per position.  GN_ONE: a thread's channels are
// of one group and one item.  Otherwise an item per channel, and GN_SPACED leaves a word out after every VEC of them: neighbouring
// lanes write an odd distance apart, where eight of them meet in every bank that an access touches if the items are GN_DENSE, but
// write single words, and reading takes more arithmetic.  Four items per channel (the statistics with their range) are 3 to 7 %
// of the call faster spaced, the two of the backward pass 1 to 6 %; the one or two of k_gn_slab 8 to 10 % slower, two without a
// range 1 %.
enum GnItems { GN_ONE, GN_DENSE, GN_SPACED };
template <int ITEMS, int VEC>
__device__ __forceinline__ uint32_t gn_item(uint32_t i) {   // vector (GN_ONE) or channel i of the set
  return i + (ITEMS == GN_SPACED && VEC > 1 ? i / VEC : 0u);
}
template <int ITEMS, int VEC>
__device__ __forceinline__ uint32_t gn_pitch(const GnShape& p) {
  return ITEMS == GN_ONE ? p.set_vecs : gn_item<ITEMS, VEC>(p.set_groups * p.dim);
}
template <int ITEMS, int VEC>
__device__ __forceinline__ void gn_deposit(float* items, const GnShape& p, const GnLane& l, const float (&v)[VEC]) {
  if (!l.live) return;
  float* const row = items + l.row * gn_pitch<ITEMS, VEC>(p);
  if constexpr (ITEMS == GN_ONE) {
    float s = v[0];
#pragma unroll
    for (int e = 1; e < VEC; ++e) s += v[e];
    row[l.vec] = s;
  } else {
#pragma unroll
    for (int e = 0; e < VEC; ++e) row[gn_item<ITEMS, VEC>(l.col + e)] = v[e];
  }
}
template <int ITEMS, int VEC>
__device__ __forceinline__ void gn_deposit_max(float* items, const GnShape& p, const GnLane& l, const float (&v)[VEC]) {
  if constexpr (ITEMS == GN_ONE) {
    float s = v[0];
#pragma unroll
    for (int e = 1; e < VEC; ++e) s = fmaxf(s, v[e]);
    if (l.live) items[l.row * p.set_vecs + l.vec] = s;
  } else {
    gn_deposit<ITEMS, VEC>(items, p, l, v);
  }
}

// 1 << fold_log2 lanes per group run through its items, group by group where there are more groups than such lane sets:
// f(group, lane among them, first item, items a position has of the group), called by whole wavefronts (with the last group again
// where lanes are left over).
template <int ITEMS, int VEC, typename F>
__device__ __forceinline__ void gn_groups(const GnShape& p, F&& f) {
  const uint32_t lanes = 1u << p.fold_log2, sets = blockDim.x >> p.fold_log2;
  const uint32_t per = ITEMS == GN_ONE ? p.dim / VEC : p.dim;
  for (uint32_t g0 = 0; g0 < p.set_groups; g0 += sets) {
    const uint32_t g = g0 + (threadIdx.x >> p.fold_log2), lane = threadIdx.x & (lanes - 1u);
    const uint32_t gc = min(g, p.set_groups - 1u);
    f(gc, lane, lane == 0 && g < p.set_groups, gc * per, per);
  }
}
// sum (or maximum) of a group's items
template <int ITEMS, int VEC, typename OP>
__device__ __forceinline__ float gn_fold(const float* items, const GnShape& p, uint32_t lane, uint32_t first, uint32_t per) {
  float a = 0.0f;
  const uint32_t n = p.rows_at_once * per, lanes = 1u << p.fold_log2;
#pragma unroll 4
  for (uint32_t i = lane; i < n; i += lanes) {
    const uint32_t row = fast_div(i, p.div_per);
    a = OP::apply(a, items[row * gn_pitch<ITEMS, VEC>(p) + gn_item<ITEMS, VEC>(first + (i - row * per))]);
  }
  return group_allreduce<OP>(a, (int)lanes);
}

}  // namespace fsk
