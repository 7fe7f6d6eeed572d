// Dropout with what stands beside it, element by element:
//   forward   y = dropout(act(x + bias)) + residual      (bias, activation and residual where there are any)
//   backward  dx = dropout(dy) * act'(x + bias)
// A thread takes eight neighbouring columns of a row, the numbers of one call of the generator, and nobody else stores its elements: an
// output may be one of the inputs' own memory.
// Memory bounds it, the generator is hidden behind 16-bit traffic: bf16 [16384,4096] with bias and residual 62.8 us, with gelu's slope 62.9
// (6.4 TB/s).  A launch of [64,128] takes 1.8 us.
#include <hip/hip_runtime.h>

#include "activation.hpp"
#include "kernel_table.hpp"
#include "vec_access.hpp"

namespace fsk {
using namespace fs;

// Eight elements of T as one or two vectors.
template <typename T> struct Eight {
  static constexpr int VEC = Elem<T>::VEC, N = 8 / VEC;
  typename VecIo<T, VEC>::Raw w[N];
  template <bool STREAM> __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = VecIo<T, VEC>::template load<STREAM>(p + i * VEC);
  }
  __device__ __forceinline__ void widen(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float part[VEC];
      VecIo<T, VEC>::widen(w[i], part);
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[i * VEC + e] = part[e];
    }
  }
  __device__ __forceinline__ static void store(T* p, const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float part[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) part[e] = v[i * VEC + e];
      VecIo<T, VEC>::store(p + i * VEC, part);
    }
  }
};

// x with its bias, through the activation and the dropout, and what `other` (residual or incoming gradient) makes of it
template <int ACT, bool SLOPE, bool OTHER>
__device__ __forceinline__ void dropped(float (&x)[8], const float (&bias)[8], const float (&other)[8], const uint32_t (&numbers)[4], uint32_t threshold,
                                        float scale) {
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] += bias[e];
  if constexpr (SLOPE) {
    float d[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) d[e] = other[e];
    drop_apply<8>(numbers, threshold, scale, d);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = d[e] * activation_slope<ACT>(x[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = activate<ACT>(x[e]);
    drop_apply<8>(numbers, threshold, scale, x);
    if constexpr (OTHER) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] += other[e];
    }
  }
}

// The values of v from place `at` on, 1 to 7, to their places behind y: one, two and four at once.
template <typename T>
__device__ __forceinline__ void store_last(T* y, uint32_t at, const float (&v)[8]) {
  if (at & 1u) {
    store1(y + at, pick(at & 4u, pick(at & 2u, v[7], v[5]), pick(at & 2u, v[3], v[1])));
    ++at;
  }
  if (at & 2u) {
    store1(y + at, pick(at & 4u, v[6], v[2]));
    store1(y + at + 1u, pick(at & 4u, v[7], v[3]));
    at += 2u;
  }
  if (at == 4u) {
    const float four[4] = {v[4], v[5], v[6], v[7]};
    VecIo<T, 4>::store(y + 4, four);
  }
}

// RAGGED: rows are no multiple of eight columns.  The last group of a row is shorter: it is read from the row's last eight elements on, its
// numbers moved up to their elements' places, and of what it computes only its own elements are stored (those in front are another
// thread's, which may have stored them already).  One path for all lanes: nearly every wavefront has the end of a row in it, and a second
// path for those lanes, element by element, took 42 us where one takes 25 to 30 (bf16 [44235,653], bias and gelu).
template <typename T, int ACT, bool SLOPE, bool OTHER, bool RAGGED, bool STREAM>
__global__ void __launch_bounds__(256) k_dropout(const T* x, const T* bias, const T* other, const void* state, T* y, uint32_t rows, uint32_t cols,
                                                 uint32_t threshold, uint32_t sequence, float scale, uint32_t groups_d, uint32_t groups_m,
                                                 uint32_t groups_s) {
  const FastDiv groups = {groups_d, groups_m, groups_s};
  const uint32_t i = blockIdx.x * 256u + threadIdx.x;
  if (i >= rows * groups_d) return;
  uint32_t numbers[4];
  float vx[8], vb[8], vo[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) vb[e] = vo[e] = 0.0f;
  uint32_t col = 0, early = 0;
  size_t at = (size_t)i * 8u;
  if (RAGGED || bias) {
    const uint32_t row = fast_div(i, groups);
    col = (i - row * groups_d) * 8u;
    if (RAGGED && col + 8u > cols) early = col + 8u - cols;
    at = (size_t)row * cols + col;
  }
  if (RAGGED && cols < 8u) {   // (element by element)
    drop_numbers<8, true>(drop_key(state), sequence, i, 0u, numbers);
#pragma unroll
    for (uint32_t e = 0; e < 8u; ++e) {
      const bool here = e < cols;
      vx[e] = here ? load1(x + at + e) : 0.0f;
      if constexpr (OTHER) vo[e] = here ? load1(other + at + e) : 0.0f;
      vb[e] = here && bias ? load1(bias + e) : 0.0f;
    }
    dropped<ACT, SLOPE, OTHER>(vx, vb, vo, numbers, threshold, scale);
#pragma unroll
    for (uint32_t e = 0; e < 8u; ++e)
      if (e < cols) store1(y + at + e, vx[e]);
    return;
  }
  if constexpr (RAGGED) col -= early, at -= early;
  Eight<T> rx, rb, ro;
  rx.template load<STREAM>(x + at);
  if constexpr (OTHER) ro.template load<STREAM>(other + at);
  if (bias) {
    rb.template load<false>(bias + col);
    rb.widen(vb);
  }
  drop_numbers<8, true>(drop_key(state), sequence, i, 0u, numbers);
  if constexpr (RAGGED) {   // up by `early` halves of a word
    uint32_t n[4];
#pragma unroll
    for (int k = 3; k >= 0; --k) n[k] = pick(early & 4u, k >= 2 ? numbers[k & 1] : 0u, numbers[k]);
#pragma unroll
    for (int k = 3; k >= 0; --k) n[k] = pick(early & 2u, k >= 1 ? n[k > 0 ? k - 1 : 0] : 0u, n[k]);
#pragma unroll
    for (int k = 3; k >= 0; --k) n[k] = pick(early & 1u, n[k] << 16 | (k >= 1 ? n[k > 0 ? k - 1 : 0] >> 16 : 0u), n[k]);
#pragma unroll
    for (int k = 0; k < 4; ++k) numbers[k] = n[k];
  }
  rx.widen(vx);
  if constexpr (OTHER) ro.widen(vo);
  dropped<ACT, SLOPE, OTHER>(vx, vb, vo, numbers, threshold, scale);
  if (!RAGGED || early == 0u) Eight<T>::store(y + at, vx);
  else store_last(y + at, early, vx);
}

}  // namespace fsk

namespace fs {
using namespace fsk;

namespace {
template <typename T, int ACT, bool SLOPE, bool OTHER>
const void* form_sym(const DropoutP& p) {
  if (p.cols % 8u != 0) return p.stream ? (const void*)k_dropout<T, ACT, SLOPE, OTHER, true, true> : (const void*)k_dropout<T, ACT, SLOPE, OTHER, true, false>;
  return p.stream ? (const void*)k_dropout<T, ACT, SLOPE, OTHER, false, true> : (const void*)k_dropout<T, ACT, SLOPE, OTHER, false, false>;
}
template <typename T, int ACT>
const void* act_sym(const DropoutP& p, bool other) {
  if constexpr (ACT != ACT_NONE)
    if (p.slope) return form_sym<T, ACT, true, true>(p);
  return other ? form_sym<T, ACT, false, true>(p) : form_sym<T, ACT, false, false>(p);
}
template <typename T>
const void* type_sym(const DropoutP& p, bool other) {
  switch (p.act) {
    case ACT_NONE: return act_sym<T, ACT_NONE>(p, other);
    case ACT_GELU: return act_sym<T, ACT_GELU>(p, other);
    case ACT_SILU: return act_sym<T, ACT_SILU>(p, other);
    default: return nullptr;
  }
}
}  // namespace

const void* dropout_kernel_symbol(int32_t, const KernelArgs& a) {
  const DropoutP& p = a.u.dropout;
  switch (p.in_dt) {
    case DT_F32: return type_sym<float>(p, p.has_other != 0);
    case DT_F16: return type_sym<f16_t>(p, p.has_other != 0);
    case DT_BF16: return type_sym<bf16_t>(p, p.has_other != 0);
    default: return nullptr;
  }
}

}  // namespace fs
