// Rotary positions of one or two tensors (queries and keys) that share their positions.
// A workgroup takes p_slots positions and h_tile of the rows at each.  Its angles depend on the positions alone, so each is formed once, by
// one thread, and handed round through LDS, the loads of a thread's rows on their way meanwhile; a thread takes the same step of 1, 2, 3 or
// 5 rows at one position, whose angles it keeps in registers.
// Memory bounds it (n elements read, n written), as long as angles are few beside elements: an angle is about 60 operations, 20 of them in
// 64 bits.  bf16 queries and keys [2,8192,32+8,128] with three axes and the head split: 59 us, 5.7 TB/s (a plain copy of as much 53); every
// thread forming its own angles 65.  Pairs that stand side by side 56.  One token of 16 sequences: 3.2 to 3.8 us, the chain of one workgroup.
#include <hip/hip_runtime.h>

#include "kernel_table.hpp"
#include "rotary.hpp"
#include "vec_access.hpp"

namespace fsk {
using namespace fs;

// First element of row h of those at a position, behind the position's own, in the second tensor or the first.  Both tensors' strides
// are read and one is taken: an index that differs from lane to lane would fetch them from the arguments' memory lane by lane.
template <bool LINES>
__device__ __forceinline__ uint32_t shared_row(const RotaryShape& s, bool second, uint32_t h, bool out) {
  const RotaryRows &t = s.t[0], &w = s.t[1];
  if constexpr (LINES) return h * (out ? (second ? w.line_out : t.line_out) : (second ? w.line_in : t.line_in));
  const uint32_t b0 = fast_div(h, t.div[0]), b1 = fast_div(h, w.div[0]), b = second ? b1 : b0, h2 = h - (second ? b1 * w.div[0].d : b0 * t.div[0].d);
  const uint32_t a0 = fast_div(b, t.div[1]), a1 = fast_div(b, w.div[1]), h0 = second ? a1 : a0, h1 = b - (second ? a1 * w.div[1].d : a0 * t.div[1].d);
  if (out) return h0 * (second ? w.out_stride[0] : t.out_stride[0]) + h1 * (second ? w.out_stride[1] : t.out_stride[1]) + h2 * (second ? w.out_stride[2] : t.out_stride[2]);
  return h0 * (second ? w.in_stride[0] : t.in_stride[0]) + h1 * (second ? w.in_stride[1] : t.in_stride[1]) + h2 * (second ? w.in_stride[2] : t.in_stride[2]);
}

// A step of a row: its accesses' first elements and its first pair, or kCopies behind the pairs.  The last step of a part of the row
// starts early where the part is no multiple of an access.
struct RotaryStep { uint32_t a, b, pair; };
constexpr uint32_t kCopies = 0xFFFFFFFFu;
template <int VEC, bool INTERLEAVED>
__device__ __forceinline__ RotaryStep rotary_step(const RotaryShape& s, uint32_t unit) {
  const uint32_t pairs = s.angles.pairs;
  const bool copies = unit >= s.rot_units;
  const uint32_t rest = min(2u * pairs + (unit - s.rot_units) * VEC, s.dim - VEC);   // (a short part: some of what was turned in front of it)
  uint32_t a, b, pair;
  if constexpr (!INTERLEAVED) pair = a = min(unit * VEC, pairs - VEC), b = a + pairs;
  else if constexpr (VEC == 1) pair = unit, a = 2u * unit, b = a + 1u;
  else a = b = min(unit * VEC, 2u * pairs - VEC), pair = a / 2u;
  return RotaryStep{copies ? rest : a, copies ? rest : b, copies ? kCopies : pair};
}

// PAIRED: elements (i, i + pairs), or single accesses: a step is one access at each of them.  Otherwise a step is one access with
// whole pairs in it.
template <typename T, int VEC, int U, bool INTERLEAVED, bool LINES, bool STREAM>
__global__ void __launch_bounds__(256) k_rotary(const T* x0, const T* x1, const int32_t* positions, T* y0, T* y1, const RotaryShape s) {
  extern __shared__ float2 turns[];
  constexpr bool PAIRED = !INTERLEAVED || VEC == 1;
  constexpr int PAIRS = INTERLEAVED && VEC > 1 ? VEC / 2 : VEC;   // of a step
  typedef VecIo<T, VEC> IO;
  const uint32_t tid = threadIdx.x, pairs = s.angles.pairs, tile = fast_div(blockIdx.x, s.div_h_tiles);
  const uint32_t p0 = tile * s.p_slots, h0 = (blockIdx.x - tile * s.div_h_tiles.d) * s.h_tile;
  const uint32_t h_end = min(h0 + s.h_tile, s.t[0].shared + s.t[1].shared);
  // this thread's place: a position, the first of its rows there, a step of the row
  const uint32_t slot = fast_div(tid, s.div_lanes), q = fast_div(slot, s.div_inner), inner = slot - q * s.div_inner.d;
  const uint32_t own_p = s.p_inner ? inner : q, own_h = s.p_inner ? q : inner;
  const bool works = own_p < s.p_slots && own_h < s.h_slots && p0 + own_p < s.positions;
  const uint32_t p = works ? p0 + own_p : p0;
  uint32_t in_p[2], out_p[2];
  {
    const uint32_t pq = fast_div(p, s.pos_div[0]), c2 = p - pq * s.pos_div[0].d, c0 = fast_div(pq, s.pos_div[1]), c1 = pq - c0 * s.pos_div[1].d;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      in_p[t] = c0 * s.t[t].in_stride[0] + c1 * s.t[t].in_stride[1] + c2 * s.t[t].in_stride[2];
      out_p[t] = c0 * s.t[t].out_stride[0] + c1 * s.t[t].out_stride[1] + c2 * s.t[t].out_stride[2];
    }
  }
  uint32_t unit = tid - slot * s.lanes;
  RotaryStep at = rotary_step<VEC, INTERLEAVED>(s, unit);
  typename IO::Raw ra[U], rb[U];
  // a thread's U rows, all that it has: the tile holds at most U * h_slots of them
  auto load = [&](uint32_t a, uint32_t b) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t row = min(h0 + own_h + (uint32_t)u * s.h_slots, h_end - 1u);
      const bool second = row >= s.t[0].shared;
      const T* const x = (second ? x1 : x0) + ((second ? in_p[1] : in_p[0]) + shared_row<LINES>(s, second, second ? row - s.t[0].shared : row, false));
      ra[u] = IO::template load<STREAM>(x + a);
      if constexpr (PAIRED) rb[u] = IO::template load<STREAM>(x + b);
    }
  };
  load(at.a, at.b);
  {
    // the workgroup's angles, a thread for one pair at one or more positions (a position is on its way while a speed is formed)
    const uint32_t first = fast_div(tid, s.div_pairs), at_once = pairs < 256u ? fast_div(256u, s.div_pairs) : 1u;
    const uint32_t here = min(s.p_slots, s.positions - p0);
    auto position = [&](uint32_t k, uint32_t axis) {
      const uint32_t n = p0 + min(k, here - 1u), aq = fast_div(n, s.pos_div[0]), a2 = n - aq * s.pos_div[0].d, a0 = fast_div(aq, s.pos_div[1]), a1 = aq - a0 * s.pos_div[1].d;
      return positions[(size_t)(a0 * s.pos_stride[0] + a1 * s.pos_stride[1] + a2 * s.pos_stride[2]) * s.angles.n_axes + axis];
    };
    if (first < at_once) {
      for (uint32_t i = tid - first * pairs; i < pairs; i += 256u) {
        const uint32_t axis = rotary_axis(s.angles, i);
        int32_t now = position(first, axis);
        const double speed = rotary_speed(s.angles, i, axis);
        for (uint32_t k = first; k < here; k += at_once) {
          const int32_t next = position(k + at_once, axis);
          float2 w;
          rotary_turn((double)now * speed, s.angles.inverse != 0, w.x, w.y);
          turns[k * pairs + i] = w;
          now = next;
        }
      }
    }
    __syncthreads();
  }
  for (;;) {   // (once, but for rows of more steps than threads)
    const uint32_t pair = at.pair;
    float c[PAIRS], d[PAIRS];   // a thread's rows are all at one position: its angles stay in registers
#pragma unroll
    for (int e = 0; e < PAIRS; ++e) {
      const float2 w = turns[(p - p0) * pairs + (pair == kCopies ? 0u : pair + (uint32_t)e)];
      c[e] = w.x;
      d[e] = w.y;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t row = h0 + own_h + (uint32_t)u * s.h_slots;
      if (!works || row >= h_end) continue;
      const bool second = row >= s.t[0].shared;
      T* const y = (second ? y1 : y0) + ((second ? out_p[1] : out_p[0]) + shared_row<LINES>(s, second, second ? row - s.t[0].shared : row, true));
      float va[VEC], vb[VEC];
      IO::widen(ra[u], va);
      if constexpr (PAIRED) {
        IO::widen(rb[u], vb);
        if (pair != kCopies) {
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const float v = va[e], w = vb[e];
            va[e] = v * c[e] - w * d[e];
            vb[e] = w * c[e] + v * d[e];
          }
          IO::store(y + at.b, vb);
        }
      } else if (pair != kCopies) {
#pragma unroll
        for (int e = 0; e < VEC; e += 2) {
          const float v = va[e], w = va[e + 1];
          va[e] = v * c[e / 2] - w * d[e / 2];
          va[e + 1] = w * c[e / 2] + v * d[e / 2];
        }
      }
      if (VEC > 1 && pair == kCopies && s.short_rest) {   // fewer elements than an access: one by one
#pragma unroll
        for (int e = 0; e < VEC; ++e)
          if (e + (int)s.short_rest >= VEC) store1(y + at.a + e, va[e]);
      } else {
        IO::store(y + at.a, va);
      }
    }
    unit += s.lanes;
    if (unit >= s.units) break;
    at = rotary_step<VEC, INTERLEAVED>(s, unit);
    load(at.a, at.b);
  }
}

}  // namespace fsk

namespace fs {
using namespace fsk;

namespace {
template <typename T, int VEC, bool INTERLEAVED, bool LINES, bool S>
const void* steps_sym(int iter) {
  switch (iter) {
    case 1: return (const void*)k_rotary<T, VEC, 1, INTERLEAVED, LINES, S>;
    case 2: return (const void*)k_rotary<T, VEC, 2, INTERLEAVED, LINES, S>;
    case 3: return (const void*)k_rotary<T, VEC, 3, INTERLEAVED, LINES, S>;
    case 5: return (const void*)k_rotary<T, VEC, 5, INTERLEAVED, LINES, S>;
    default: return nullptr;
  }
}
template <typename T, int VEC, bool S>
const void* layout_sym(const RotaryP& p) {
  if (p.s.lines) return p.interleaved ? steps_sym<T, VEC, true, true, S>(p.iter) : steps_sym<T, VEC, false, true, S>(p.iter);
  return p.interleaved ? steps_sym<T, VEC, true, false, S>(p.iter) : steps_sym<T, VEC, false, false, S>(p.iter);
}
template <typename T>
const void* type_sym(const RotaryP& p) {
  if (p.vec == 1) return layout_sym<T, 1, false>(p);
  if constexpr (sizeof(T) == 2)
    if (p.vec == 4) return layout_sym<T, 4, false>(p);
  return p.stream ? layout_sym<T, Elem<T>::VEC, true>(p) : layout_sym<T, Elem<T>::VEC, false>(p);
}
}  // namespace

const void* rotary_kernel_symbol(int32_t, const KernelArgs& a) {
  switch (a.u.rotary.in_dt) {
    case DT_F32: return type_sym<float>(a.u.rotary);
    case DT_F16: return type_sym<f16_t>(a.u.rotary);
    case DT_BF16: return type_sym<bf16_t>(a.u.rotary);
    default: return nullptr;
  }
}

}  // namespace fs
