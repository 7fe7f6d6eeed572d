// Rotary positions of one or two tensors (queries and keys) that share their positions.
// A workgroup takes p_tile positions and h_tile of the rows at each.  Its angles depend on the positions alone, so each is formed once, by
// one thread, and all the workgroup's rows read them from LDS; the loads of a lane's first steps are on their way meanwhile.
#include <hip/hip_runtime.h>

#include "kernel_table.hpp"
#include "rotary.hpp"
#include "vec_access.hpp"

namespace fsk {
using namespace fs;

// Where a row lies, from its number among the workgroup's.
struct RotaryRow {
  uint32_t second, in, out, p;   // second tensor?  first elements; position within the tile
  bool there;
};
__device__ __forceinline__ RotaryRow rotary_row(const RotaryShape& s, uint32_t number, uint32_t p0, uint32_t h0) {
  RotaryRow r;
  const uint32_t q = fast_div(number, s.div_inner), inner = number - q * s.div_inner.d;
  r.p = s.p_inner ? inner : q;
  uint32_t h = h0 + (s.p_inner ? q : inner), p = p0 + r.p;
  r.there = r.p < s.p_tile && h - h0 < s.h_tile && p < s.positions && h < s.t[0].shared + s.t[1].shared;
  if (!r.there) p = p0, h = h0, r.p = 0;
  r.second = h >= s.t[0].shared ? 1u : 0u;
  if (r.second) h -= s.t[0].shared;
  const uint32_t a = fast_div(p, s.pos_div[0]), p2 = p - a * s.pos_div[0].d, pa = fast_div(a, s.pos_div[1]), p1 = a - pa * s.pos_div[1].d;
  const RotaryRows& t = s.t[r.second];
  const uint32_t b = fast_div(h, t.div[0]), h2 = h - b * t.div[0].d, hb = fast_div(b, t.div[1]), h1 = b - hb * t.div[1].d;
  r.in = (pa + hb) * t.in_stride[0] + (p1 + h1) * t.in_stride[1] + (p2 + h2) * t.in_stride[2];
  r.out = (pa + hb) * t.out_stride[0] + (p1 + h1) * t.out_stride[1] + (p2 + h2) * t.out_stride[2];
  return r;
}

// PAIRED: elements (i, i + pairs), or single accesses: a step is one access at each of them.  Otherwise a step is one access with
// whole pairs in it.  The last step of a part of the row starts early where the part is no multiple of an access.
template <typename T, int VEC, int U, bool INTERLEAVED, bool STREAM>
__global__ void __launch_bounds__(256) k_rotary(const T* x0, const T* x1, const int32_t* positions, T* y0, T* y1, const RotaryShape s) {
  extern __shared__ float2 turns[];
  constexpr bool PAIRED = !INTERLEAVED || VEC == 1;
  typedef VecIo<T, VEC> IO;
  const uint32_t pairs = s.angles.pairs, tile = fast_div(blockIdx.x, s.div_h_tiles);
  const uint32_t p0 = tile * s.p_tile, h0 = (blockIdx.x - tile * s.div_h_tiles.d) * s.h_tile;
  const uint32_t items = s.p_tile * s.h_tile * s.div_units.d;
  for (uint32_t first = 0; first < items; first += 256u * U) {
    typename IO::Raw ra[U], rb[U];
    RotaryRow row[U];
    uint32_t a[U], b[U], pair[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t item = first + (uint32_t)u * 256u + threadIdx.x;
      const uint32_t number = fast_div(item, s.div_units), unit = item - number * s.div_units.d;
      row[u] = rotary_row(s, number, p0, h0);
      pair[u] = 0xFFFFFFFFu;   // a step that copies
      if (unit >= s.rot_units) {
        a[u] = b[u] = 2u * pairs + min((unit - s.rot_units) * VEC, s.dim - 2u * pairs - VEC);
      } else if constexpr (!INTERLEAVED) {
        pair[u] = a[u] = min(unit * VEC, pairs - VEC);
        b[u] = a[u] + pairs;
      } else if constexpr (VEC == 1) {
        pair[u] = unit;
        a[u] = 2u * unit;
        b[u] = a[u] + 1u;
      } else {
        a[u] = b[u] = min(unit * VEC, 2u * pairs - VEC);
        pair[u] = a[u] / 2u;
      }
      const T* const x = (row[u].second ? x1 : x0) + row[u].in;
      ra[u] = IO::template load<STREAM>(x + a[u]);
      if constexpr (PAIRED) rb[u] = IO::template load<STREAM>(x + b[u]);
    }
    if (first == 0) {
      const uint32_t here = min(s.p_tile, s.positions - p0) * pairs;
      for (uint32_t t = threadIdx.x; t < here; t += 256u) {
        const uint32_t p = t / pairs, i = t - p * pairs, at = p0 + p;
        const uint32_t q = fast_div(at, s.pos_div[0]), p2 = at - q * s.pos_div[0].d, pa = fast_div(q, s.pos_div[1]), p1 = q - pa * s.pos_div[1].d;
        const uint32_t axis = rotary_axis(s.angles, i);
        const size_t from = (size_t)(pa * s.pos_stride[0] + p1 * s.pos_stride[1] + p2 * s.pos_stride[2]) * s.angles.n_axes + axis;
        float c, d;
        rotary_turn(s.angles, i, axis, positions[from], c, d);
        turns[t] = float2{c, d};
      }
      __syncthreads();
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!row[u].there) continue;
      T* const y = (row[u].second ? y1 : y0) + row[u].out;
      float va[VEC], vb[VEC];
      IO::widen(ra[u], va);
      if constexpr (PAIRED) {
        IO::widen(rb[u], vb);
        if (pair[u] != 0xFFFFFFFFu) {
          const float2* const t = turns + row[u].p * pairs + pair[u];
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const float2 w = t[e];
            const float p = va[e], q = vb[e];
            va[e] = p * w.x - q * w.y;
            vb[e] = q * w.x + p * w.y;
          }
          IO::store(y + b[u], vb);
        }
      } else if (pair[u] != 0xFFFFFFFFu) {
        const float2* const t = turns + row[u].p * pairs + pair[u];
#pragma unroll
        for (int e = 0; e < VEC; e += 2) {
          const float2 w = t[e / 2];
          const float p = va[e], q = va[e + 1];
          va[e] = p * w.x - q * w.y;
          va[e + 1] = q * w.x + p * w.y;
        }
      }
      IO::store(y + a[u], va);
    }
  }
}

}  // namespace fsk

namespace fs {
using namespace fsk;

namespace {
template <typename T, int VEC, bool INTERLEAVED, bool S>
const void* steps_sym(int iter) {
  switch (iter) {
    case 1: return (const void*)k_rotary<T, VEC, 1, INTERLEAVED, S>;
    case 2: return (const void*)k_rotary<T, VEC, 2, INTERLEAVED, S>;
    case 4: return (const void*)k_rotary<T, VEC, 4, INTERLEAVED, S>;
    default: return nullptr;
  }
}
template <typename T, int VEC, bool S>
const void* layout_sym(const RotaryP& p) {
  return p.interleaved ? steps_sym<T, VEC, true, S>(p.iter) : steps_sym<T, VEC, false, S>(p.iter);
}
template <typename T>
const void* type_sym(const RotaryP& p) {
  if (p.vec == 1) return layout_sym<T, 1, false>(p);
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
