// Root-mean-square normalisation behind a residual connection, its result in 8 bits with a scale per row:
//   h = x,  x + bias + residual,  or  dropout(x + bias) + residual
//   r = 1 / sqrt(mean h^2 + eps),  n = h r gamma,  s = max |n| / 448 + tiny,  q = e4m3(n / s)
// A lane group or a workgroup holds the row between its sum and its quotients: what is read is read once.  The largest |n| is r times
// the largest |h gamma|, so one pass over the registers and one exchange between lanes give both the sum and the maximum.  (Taken of n itself,
// in an exchange of its own behind the sum's, the maximum would be rounded as n is, not once otherwise; that took 40.2 instead of 39.0 us at
// bf16 [8192,4096], 46.5 instead of 42.5 at [2048,16384], and r's last bit, from the order of the sum, moves as many quotients over a rounding
// border of the 8-bit format as the maximum's.)
// Memory bounds it: x and the residual read, h and q written, 7 bytes an element of 16 bits.  bf16 [8192,4096] 39.0 us, 6.0 TB/s; f16
// [8192,2048] 22.0, with bias and dropout 22.8 (5.2 TB/s; the launch's ramp is 3 of it); [8191,2050] 22 to 26, rows straddle lines.  Four
// rows of 4096: 2.5 us, the chain of load, sum, exchange, quotient.
#include <hip/hip_runtime.h>

#include "activation.hpp"
#include "kernel_table.hpp"
#include "vec_access.hpp"

namespace fsk {
using namespace fs;

enum RmsForm : int { RMS_PLAIN = 0, RMS_RESIDUAL = 1, RMS_DROPPED = 2 };   // h = x; x (+ bias) + residual; dropout(x (+ bias)) + residual

struct Rms8Args {
  uint32_t rows, cols, flags;   // flags: 1 gamma is float32 beside a 16-bit type, 2 h is rounded to that type before the norm reads it
  float eps, inv_cols, inv_max, tiny;
  uint32_t threshold, sequence;
  float scale;
};

template <typename T, int VEC>
__device__ __forceinline__ void round_to_storage(float (&v)[VEC], const T*) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      T t;
      store1(&t, v[e]);
      v[e] = load1(&t);
    }
  }
}

// VEC of the row's values from column `col` on
template <typename T, int VEC, int FORM, bool STREAM>
struct Rms8Source {
  typedef VecIo<T, VEC> IO;
  typename IO::Raw x, res, bias;
  __device__ __forceinline__ void load(const T* px, const T* pres, const T* pbias, size_t base, uint32_t col) {
    x = IO::template load<STREAM>(px + base + col);
    if constexpr (FORM != RMS_PLAIN) {
      res = IO::template load<STREAM>(pres + base + col);
      if (pbias) bias = IO::template load<false>(pbias + col);
    }
  }
  __device__ __forceinline__ void values(bool has_bias, const uint32_t (&numbers)[(VEC + 1) / 2], const Rms8Args& a, float (&h)[VEC]) const {
    IO::widen(x, h);
    if constexpr (FORM != RMS_PLAIN) {
      float t[VEC];
      if (has_bias) {
        IO::widen(bias, t);
#pragma unroll
        for (int e = 0; e < VEC; ++e) h[e] += t[e];
      }
      if constexpr (FORM == RMS_DROPPED) drop_apply<VEC>(numbers, a.threshold, a.scale, h);
      IO::widen(res, t);
#pragma unroll
      for (int e = 0; e < VEC; ++e) h[e] += t[e];
    }
    if (a.flags & 2u) round_to_storage<T, VEC>(h, (const T*)nullptr);
  }
};

// The numbers of the vector that starts at `start` of the row, or early, at `col`: its own group's, but for a row's last vector that
// starts early (in one wavefront of a row; a vector behind the row's end has none).
template <int VEC, int FORM, bool WHOLE>
__device__ __forceinline__ void row_numbers(const void* state, const Rms8Args& a, uint32_t row, uint32_t start, uint32_t col, uint32_t (&n)[(VEC + 1) / 2]) {
  if constexpr (FORM == RMS_DROPPED) {
    const DropKey key = drop_key(state);
    const uint32_t first = row * ((a.cols + 7u) / 8u);
    if constexpr (WHOLE) {
      drop_numbers<VEC, true>(key, a.sequence, first, col, n);
    } else {
      if (start == col) drop_numbers<VEC, true>(key, a.sequence, first, col, n);
      else if (start < a.cols) drop_numbers<VEC, false>(key, a.sequence, first, col, n);
    }
  }
}

template <typename T, int VEC>
__device__ __forceinline__ void load_gains(const void* gamma, uint32_t flags, uint32_t col, float (&g)[VEC]) {
  if (sizeof(T) == 4 || !(flags & 1u)) {
    VecIo<T, VEC>::widen(VecIo<T, VEC>::template load<false>(static_cast<const T*>(gamma) + col), g);
  } else if constexpr (VEC == 1) {
    g[0] = static_cast<const float*>(gamma)[col];
  } else {
#pragma unroll
    for (int i = 0; i < VEC; i += 4) {
      float part[4];
      VecIo<float, 4>::widen(VecIo<float, 4>::load<false>(static_cast<const float*>(gamma) + col + i), part);
#pragma unroll
      for (int e = 0; e < 4; ++e) g[i + e] = part[e];
    }
  }
}

// Whether max |h gamma| has lost what n = h r gamma keeps: beyond the range, or below the normal one, where a product has fewer bits
// than n or none (and where all are 0, r may be infinite).  A NaN has not come through.
__device__ __forceinline__ bool left_range(float most) { return !(most < __builtin_inff() && most >= 1.17549435e-38f); }

// The row's sum of squares and largest magnitude from the lanes': over a lane group, or over the workgroup through LDS.
template <bool BLOCK>
__device__ __forceinline__ void rms8_join(float& sum, float& most, float (*slot)[2], uint32_t lanes) {
  // A lane's only square, fused into the first addition, would go in unrounded there and rounded into its neighbours' sums: the lanes of a
  // row would normalise by different r.  (No instruction.)
  asm volatile("" : "+v"(sum));
  if constexpr (BLOCK) {
    sum = group_allreduce<OpSum>(sum, kWave);
    most = group_allreduce<OpMax>(most, kWave);
    const uint32_t wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    if ((threadIdx.x & 63u) == 0u) slot[wave][0] = sum, slot[wave][1] = most;
    __syncthreads();
    sum = slot[0][0], most = slot[0][1];
    for (uint32_t w = 1; w < waves; ++w) sum += slot[w][0], most = fmaxf(most, slot[w][1]);
  } else {
    sum = group_allreduce<OpSum>(sum, (int)lanes);
    most = group_allreduce<OpMax>(most, (int)lanes);
  }
}

// BLOCK: the whole workgroup on a row, otherwise 1 << lanes_log2 lanes; K vectors per lane.  The last vector of a row whose length is
// no multiple of VEC starts early, at the row's last VEC elements; what the vector before it holds as well counts once in the sum and
// is written twice, the same.
// WHOLE: the length is a multiple of VEC.  A dropout's numbers need nothing of the row, so they are drawn while its loads are on their way.
template <typename T, int VEC, int K, int FORM, bool BLOCK, bool STREAM, bool WHOLE>
__global__ void __launch_bounds__(BLOCK ? 1024 : 256) k_rmsnorm8(const T* x, const T* res, const void* gamma, uint32_t rows, uint32_t cols, const T* bias,
                                                               const void* state, T* h_out, T* n_out, e4m3_t* q_out, float* scales, float* deviations,
                                                               int32_t lanes_log2, uint32_t flags, float eps, float inv_cols, float inv_max, float tiny,
                                                               uint32_t threshold, uint32_t sequence, float drop_scale) {
  __shared__ float slot[2][16][2];
  const Rms8Args a = {rows, cols, flags, eps, inv_cols, inv_max, tiny, threshold, sequence, drop_scale};
  const uint32_t L = BLOCK ? blockDim.x : 1u << lanes_log2;
  const uint32_t lane = BLOCK ? threadIdx.x : threadIdx.x & (L - 1u);
  const uint32_t row = BLOCK ? blockIdx.x : blockIdx.x * (256u >> lanes_log2) + (threadIdx.x >> lanes_log2);
  const uint32_t r = min(row, rows - 1u);
  const size_t base = (size_t)r * cols;
  Rms8Source<T, VEC, FORM, STREAM> source[K];
  uint32_t col[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    col[k] = min((lane + (uint32_t)k * L) * VEC, cols - VEC);
    source[k].load(x, res, bias, base, col[k]);
  }
  uint32_t numbers[K][(VEC + 1) / 2] = {};
#pragma unroll
  for (int k = 0; k < K; ++k) row_numbers<VEC, FORM, WHOLE>(state, a, r, (lane + (uint32_t)k * L) * VEC, col[k], numbers[k]);
  float h[K][VEC], g[K][VEC];
#pragma unroll
  for (int k = 0; k < K; ++k) load_gains<T, VEC>(gamma, flags, col[k], g[k]);
  float sum = 0.0f, most = 0.0f;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    source[k].values(bias != nullptr, numbers[k], a, h[k]);
    const uint32_t again = (lane + (uint32_t)k * L) * VEC - col[k];   // elements that another vector holds too (VEC and more: all)
    if (again >= (uint32_t)VEC) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) h[k][e] = 0.0f;
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      sum += WHOLE || (uint32_t)e >= again ? h[k][e] * h[k][e] : 0.0f;
      most = fmaxf(most, __builtin_fabsf(h[k][e] * g[k][e]));
    }
  }
  rms8_join<BLOCK>(sum, most, slot[0], L);
  const float rr = fast_rsqrt(sum * inv_cols + eps);
  float largest = most * rr;
  // Where the products with the gains have left the range, or the row holds an infinity, the maximum is taken of n itself, as it is
  // defined.  (All lanes of a wavefront take part in the exchange, whosever row it is for.)
  if (__any(left_range(most))) {
    float m = 0.0f, none = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int e = 0; e < VEC; ++e) m = fmaxf(m, __builtin_fabsf(h[k][e] * rr * g[k][e]));
    rms8_join<BLOCK>(none, m, slot[1], L);
    if (left_range(most)) largest = rr == rr ? m : rr;
  }
  const Divisor s(scale_of(largest, inv_max, tiny));
  if (row >= rows) return;
  if (lane == 0) {
    scales[row] = s.s;
    if (deviations) deviations[row] = rr;
  }
#pragma unroll
  for (int k = 0; k < K; ++k) {
    if ((lane + (uint32_t)k * L) * VEC < cols) {
      if (h_out) VecIo<T, VEC>::store(h_out + base + col[k], h[k]);
      float n[VEC], d[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        n[e] = h[k][e] * rr * g[k][e];
        d[e] = s.divide(n[e]);
      }
      VecIo<e4m3_t, VEC>::store(q_out + base + col[k], d);
      if (n_out) VecIo<T, VEC>::store(n_out + base + col[k], n);
    }
  }
}

// Rows that no workgroup can hold: read twice, once for the sum and the maximum and once for the quotients.  A lane adds the sums of its
// vectors up in 64 bits: one float32 for 2^14 squares and more, a lane's share of 2^24 columns, was off by 1e-4 of itself (and the lanes
// by the same where values are alike).
template <typename T, int VEC, int FORM>
__global__ void __launch_bounds__(1024) k_rmsnorm8_long(const T* x, const T* res, const void* gamma, uint32_t rows, uint32_t cols, const T* bias,
                                                        const void* state, T* h_out, T* n_out, e4m3_t* q_out, float* scales, float* deviations, int32_t,
                                                        uint32_t flags, float eps, float inv_cols, float inv_max, float tiny, uint32_t threshold,
                                                        uint32_t sequence, float drop_scale) {
  __shared__ float slot[2][16][2];
  const Rms8Args a = {rows, cols, flags, eps, inv_cols, inv_max, tiny, threshold, sequence, drop_scale};
  const uint32_t row = blockIdx.x;
  const size_t base = (size_t)row * cols;
  auto values = [&](uint32_t start, uint32_t col, float (&h)[VEC], float (&g)[VEC]) {
    Rms8Source<T, VEC, FORM, false> source;
    source.load(x, res, bias, base, col);
    uint32_t numbers[(VEC + 1) / 2] = {};
    row_numbers<VEC, FORM, false>(state, a, row, start, col, numbers);
    load_gains<T, VEC>(gamma, flags, col, g);
    source.values(bias != nullptr, numbers, a, h);
  };
  double squares = 0.0;
  float most = 0.0f;
  for (uint32_t c = threadIdx.x * VEC; c < cols; c += 1024u * VEC) {
    float h[VEC], g[VEC], part = 0.0f;
    const uint32_t col = min(c, cols - VEC);
    values(c, col, h, g);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      part += col + (uint32_t)e >= c ? h[e] * h[e] : 0.0f;
      most = fmaxf(most, __builtin_fabsf(h[e] * g[e]));
    }
    squares += (double)part;
    if (h_out) VecIo<T, VEC>::store(h_out + base + col, h);
  }
  float sum = (float)squares;
  rms8_join<true>(sum, most, slot[0], 1024u);
  const float rr = fast_rsqrt(sum * inv_cols + eps);
  float largest = most * rr;
  if (left_range(most)) {   // (the whole workgroup's: see k_rmsnorm8)
    float m = 0.0f, none = 0.0f;
    for (uint32_t c = threadIdx.x * VEC; c < cols; c += 1024u * VEC) {
      float h[VEC], g[VEC];
      values(c, min(c, cols - VEC), h, g);
#pragma unroll
      for (int e = 0; e < VEC; ++e) m = fmaxf(m, __builtin_fabsf(h[e] * rr * g[e]));
    }
    rms8_join<true>(none, m, slot[1], 1024u);
    largest = rr == rr ? m : rr;
  }
  const Divisor s(scale_of(largest, inv_max, tiny));
  if (threadIdx.x == 0) {
    scales[row] = s.s;
    if (deviations) deviations[row] = rr;
  }
  for (uint32_t c = threadIdx.x * VEC; c < cols; c += 1024u * VEC) {
    float h[VEC], g[VEC], d[VEC];
    const uint32_t col = min(c, cols - VEC);
    values(c, col, h, g);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      h[e] = h[e] * rr * g[e];
      d[e] = s.divide(h[e]);
    }
    VecIo<e4m3_t, VEC>::store(q_out + base + col, d);
    if (n_out) VecIo<T, VEC>::store(n_out + base + col, h);
  }
}

}  // namespace fsk

namespace fs {
using namespace fsk;

namespace {
template <typename T, int VEC, int FORM, bool S, bool WHOLE>
const void* shape_sym(int32_t kernel, int vecs) {
  if (kernel == K_RMS8_LONG) return VEC > 1 ? (const void*)k_rmsnorm8_long<T, VEC, FORM> : nullptr;
  if constexpr (VEC == 1) return kernel == K_RMS8_WAVE && vecs == 1 ? (const void*)k_rmsnorm8<T, 1, 1, FORM, false, S, true> : nullptr;
  else if (kernel == K_RMS8_WAVE) {
    switch (vecs) {
      case 1: return (const void*)k_rmsnorm8<T, VEC, 1, FORM, false, S, WHOLE>;
      case 2: return (const void*)k_rmsnorm8<T, VEC, 2, FORM, false, S, WHOLE>;
      case 4: return (const void*)k_rmsnorm8<T, VEC, 4, FORM, false, S, WHOLE>;
      case 8: return (const void*)k_rmsnorm8<T, VEC, 8, FORM, false, S, WHOLE>;
    }
  } else {
    switch (vecs) {
      case 1: return (const void*)k_rmsnorm8<T, VEC, 1, FORM, true, S, WHOLE>;
      case 2: return (const void*)k_rmsnorm8<T, VEC, 2, FORM, true, S, WHOLE>;
      case 4: return (const void*)k_rmsnorm8<T, VEC, 4, FORM, true, S, WHOLE>;
    }
  }
  return nullptr;
}
template <typename T, int VEC, int FORM, bool S>
const void* whole_sym(int32_t kernel, const RmsNorm8P& p) {
  return p.cols % VEC == 0 ? shape_sym<T, VEC, FORM, S, true>(kernel, p.vecs_per_lane) : shape_sym<T, VEC, FORM, S, false>(kernel, p.vecs_per_lane);
}
template <typename T, int VEC, bool S>
const void* form_sym(int32_t kernel, const KernelArgs& a) {
  const RmsNorm8P& p = a.u.rms8;
  if (p.form == RMS_PLAIN) return whole_sym<T, VEC, RMS_PLAIN, S>(kernel, p);
  return p.form == RMS_DROPPED ? whole_sym<T, VEC, RMS_DROPPED, S>(kernel, p) : whole_sym<T, VEC, RMS_RESIDUAL, S>(kernel, p);
}
template <typename T>
const void* type_sym(int32_t kernel, const KernelArgs& a) {
  const RmsNorm8P& p = a.u.rms8;
  if (p.vec == 1) return form_sym<T, 1, false>(kernel, a);
  return p.stream ? form_sym<T, Elem<T>::VEC, true>(kernel, a) : form_sym<T, Elem<T>::VEC, false>(kernel, a);
}
}  // namespace

const void* rmsnorm8_kernel_symbol(int32_t kernel, const KernelArgs& a) {
  switch (a.u.rms8.dt) {
    case DT_F32: return type_sym<float>(kernel, a);
    case DT_F16: return type_sym<f16_t>(kernel, a);
    case DT_BF16: return type_sym<bf16_t>(kernel, a);
    default: return nullptr;
  }
}

}  // namespace fs
