// Backward pass of group normalisation with an activation.  With xh the normalised values ((x - mean) rstd, or an 8-bit
// checkpoint times its scale), dz = dy act'(xh gamma + beta) and, per batch entry and channel,
//     A = sum over positions of dz,   B = sum over positions of dz xh
// everything else follows: dbeta = sum_n A, dgamma = sum_n B, and for a group's n values
//     m1 = sum_d gamma A / n,   m2 = sum_d gamma B / n,   dx = (gamma dz - m1 - xh m2) rstd.
// A workgroup that holds a set's values (k_gn_bwd_slab) reads them once; otherwise a first launch gathers A and B per chunk of
// positions, a second adds the chunks and makes the group means, a third reads the values again.  K_COLFOLD adds up the batch.
#include <hip/hip_runtime.h>

#include "group_norm.hpp"
#include "kernel_table.hpp"

namespace fsk {
using namespace fs;

// The normalised values' storage: their 8-bit checkpoint, or the input.
template <typename T, bool FROM8> struct GnValue { typedef T type; };
template <typename T> struct GnValue<T, true> { typedef e4m3_t type; };

// What a thread knows of its channels: xh = (v - shift) * scale.
template <typename T, int VEC, bool FROM8>
struct GnChannels {
  float shift[VEC], scale[VEC], ga[VEC], be[VEC];
  // `centre`: means, or the checkpoint's scales
  __device__ __forceinline__ void load(const GnShape& p, const GnLane& l, uint32_t n, uint32_t set, const float* centre, const float* rstd,
                                       const T* gamma, const T* beta) {
    const uint32_t c = set * p.set_groups * p.dim + l.col, g0 = n * p.groups;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const uint32_t g = g0 + fast_div(c + e, p.div_dim);
      shift[e] = FROM8 ? 0.0f : centre[g];
      scale[e] = FROM8 ? centre[g] : rstd[g];
    }
    VecIo<T, VEC>::widen(VecIo<T, VEC>::template load<false>(gamma + c), ga);
    if (beta) VecIo<T, VEC>::widen(VecIo<T, VEC>::template load<false>(beta + c), be);
  }
  __device__ __forceinline__ float normal(float v, int e) const { return FROM8 ? v * scale[e] : (v - shift[e]) * scale[e]; }
  template <int ACT>
  __device__ __forceinline__ float dz(float xh, float dy, int e) const {
    if constexpr (ACT == ACT_NONE) return dy;
    else return dy * activation_slope<ACT>(__builtin_fmaf(xh, ga[e], be[e]));
  }
};

// Sums over the workgroup's positions of what every thread has gathered per channel: channel c of the set to out[c], by
// 1 << fold_log2 lanes each.  `items`: rows_at_once * width floats of LDS.
template <int VEC>
__device__ __forceinline__ void gn_channel_sums(float* items, const GnShape& p, const GnLane& l, const float (&v)[VEC], float* sums, float* out) {
  const uint32_t width = p.set_groups * p.dim, lanes = 1u << p.fold_log2, lane = threadIdx.x & (lanes - 1u);
  gn_deposit<false, VEC>(items, p, l, v);
  __syncthreads();
  for (uint32_t c0 = 0; c0 < width; c0 += blockDim.x >> p.fold_log2) {
    const uint32_t c = c0 + (threadIdx.x >> p.fold_log2), cc = min(c, width - 1u);
    float a = 0.0f;
#pragma unroll 4
    for (uint32_t r = lane; r < p.rows_at_once; r += lanes) a += items[r * width + cc];
    a = group_allreduce<OpSum>(a, (int)lanes);
    if (lane == 0 && c < width) {
      sums[c] = a;
      out[c] = a;
    }
  }
  __syncthreads();
}

// ---- one launch (and the fold over the batch) --------------------------------------------------------------------------------
template <typename T, int VEC, int K, int ACT, bool FROM8, int NT>
__global__ void __launch_bounds__(NT) k_gn_bwd_slab(const typename GnValue<T, FROM8>::type* x, const float* centre, const float* rstd, const T* gamma,
                                                    const T* beta, const T* dy, T* dx, float* sums, const GnShape p) {
  typedef typename GnValue<T, FROM8>::type X;
  extern __shared__ __align__(16) float lds[];
  const uint32_t width = p.set_groups * p.dim;
  float* const items = lds;
  float* const sum_a = lds + p.rows_at_once * width;
  float* const sum_b = sum_a + width;
  float* const means = sum_b + width;   // [set_groups][2]
  const uint32_t b = gn_block(p.batch * p.sets), n = fast_div(b, p.div_sets), set = b - n * p.sets;
  const GnLane l = gn_lane<VEC>(p);
  const size_t base = (size_t)n * p.positions * p.channels + set * width;
  const uint32_t place = l.row * p.channels + l.col, step = p.rows_at_once * p.channels, last = (p.positions - 1u) * p.channels + l.col;
  typename VecIo<X, VEC>::Raw rx[K];
  typename VecIo<T, VEC>::Raw rd[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    rx[k] = VecIo<X, VEC>::template load<false>(near_element(x + base, min(place + (uint32_t)k * step, last)));
    rd[k] = VecIo<T, VEC>::template load<false>(near_element(dy + base, min(place + (uint32_t)k * step, last)));
  }
  GnChannels<T, VEC, FROM8> ch;
  ch.load(p, l, n, set, centre, rstd, gamma, beta);
  auto valid = [&](int k) { return l.live && place + (uint32_t)k * step <= last; };
  float a[VEC], bb[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) a[e] = bb[e] = 0.0f;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    float v[VEC], d[VEC];
    again(rx[k]);
    again(rd[k]);
    VecIo<X, VEC>::widen(rx[k], v);
    VecIo<T, VEC>::widen(rd[k], d);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float xh = ch.normal(v[e], e);
      const float dz = ch.template dz<ACT>(xh, d[e], e);
      a[e] += valid(k) ? dz : 0.0f;
      bb[e] += valid(k) ? dz * xh : 0.0f;
    }
    done(a);
    done(bb);
  }
  const uint32_t pitch = p.sum_pitch;
  float* const out = sums + (size_t)n * 2u * pitch + set * width;
  gn_channel_sums<VEC>(items, p, l, a, sum_a, out);
  gn_channel_sums<VEC>(items, p, l, bb, sum_b, out + pitch);
  // a wavefront per group
  for (uint32_t g0 = 0; g0 < p.set_groups; g0 += NT / 64) {
    const uint32_t g = g0 + (threadIdx.x >> 6), gc = min(g, p.set_groups - 1u);
    float m1 = 0.0f, m2 = 0.0f;
    for (uint32_t d = threadIdx.x & 63u; d < p.dim; d += 64u) {
      const float w = load1(gamma + set * width + gc * p.dim + d);
      m1 = __builtin_fmaf(w, sum_a[gc * p.dim + d], m1);
      m2 = __builtin_fmaf(w, sum_b[gc * p.dim + d], m2);
    }
    m1 = group_allreduce<OpSum>(m1, 64);
    m2 = group_allreduce<OpSum>(m2, 64);
    if ((threadIdx.x & 63u) == 0 && g < p.set_groups) {
      means[2u * g] = m1 * p.inv_count;
      means[2u * g + 1u] = m2 * p.inv_count;
    }
  }
  __syncthreads();
  float m1[VEC], m2[VEC], r[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    const uint32_t g = fast_div(l.col + e, p.div_dim);
    m1[e] = means[2u * g];
    m2[e] = means[2u * g + 1u];
    r[e] = FROM8 ? rstd[n * p.groups + set * p.set_groups + g] : ch.scale[e];
  }
#pragma unroll
  for (int k = 0; k < K; ++k) {
    again(rx[k]);
    again(rd[k]);
    if (!valid(k)) continue;
    float v[VEC], d[VEC];
    VecIo<X, VEC>::widen(rx[k], v);
    VecIo<T, VEC>::widen(rd[k], d);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float xh = ch.normal(v[e], e);
      const float dz = ch.template dz<ACT>(xh, d[e], e);
      d[e] = (__builtin_fmaf(dz, ch.ga[e], -m1[e]) - xh * m2[e]) * r[e];
    }
    VecIo<T, VEC>::store(near_element(dx + base, place + (uint32_t)k * step), d);
  }
}

// ---- first launch of three: A and B of a chunk of positions ------------------------------------------------------------------
template <typename T, int VEC, int ACT, bool FROM8>
__global__ void __launch_bounds__(256) k_gn_bwd_sums(const typename GnValue<T, FROM8>::type* x, const float* centre, const float* rstd, const T* gamma,
                                                     const T* beta, const T* dy, float* out, const GnShape p) {
  typedef typename GnValue<T, FROM8>::type X;
  extern __shared__ __align__(16) float lds[];
  constexpr int U = 4;
  const uint32_t width = p.set_groups * p.dim;
  const uint32_t bc = fast_div(blockIdx.x, p.div_sets), set = blockIdx.x - bc * p.sets;
  const uint32_t n = fast_div(bc, p.div_chunks), chunk = bc - n * p.chunks;
  const uint32_t r0 = chunk * p.chunk_rows, r1 = min(r0 + p.chunk_rows, p.positions);
  const GnLane l = gn_lane<VEC>(p);
  float a[VEC], b[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) a[e] = b[e] = 0.0f;
  if (l.live) {
    const size_t base = (size_t)n * p.positions * p.channels + set * width + l.col;
    const uint32_t step = p.rows_at_once;
    uint32_t row = r0 + l.row;
    typename VecIo<X, VEC>::Raw nx[U], x0[U];
    typename VecIo<T, VEC>::Raw nd[U], d0[U];
    auto issue = [&]() {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const size_t at = base + min(row + u * step, r1 - 1u) * p.channels;
        nx[u] = VecIo<X, VEC>::template load<false>(x + at);
        nd[u] = VecIo<T, VEC>::template load<false>(dy + at);
      }
    };
    issue();
    GnChannels<T, VEC, FROM8> ch;
    ch.load(p, l, n, set, centre, rstd, gamma, beta);
    auto add = [&](typename VecIo<X, VEC>::Raw rx, typename VecIo<T, VEC>::Raw rd) {
      float v[VEC], d[VEC];
      VecIo<X, VEC>::widen(rx, v);
      VecIo<T, VEC>::widen(rd, d);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float xh = ch.normal(v[e], e);
        const float dz = ch.template dz<ACT>(xh, d[e], e);
        a[e] += dz;
        b[e] = __builtin_fmaf(dz, xh, b[e]);
      }
      done(a);
      done(b);
    };
    for (uint32_t all = r0 + U * step; all <= r1; all += U * step) {   // (every live thread has the positions below `all`)
#pragma unroll
      for (int u = 0; u < U; ++u) x0[u] = nx[u], d0[u] = nd[u];
      row += U * step;
      issue();
#pragma unroll
      for (int u = 0; u < U; ++u) add(x0[u], d0[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (row + u * step < r1) add(nx[u], nd[u]);
  }
  float* const to = out + (size_t)bc * 2u * p.channels + set * width;
  float* const spare = lds + p.rows_at_once * width;   // (the sums in LDS are not read here)
  gn_channel_sums<VEC>(lds, p, l, a, spare, to);
  gn_channel_sums<VEC>(lds, p, l, b, spare, to + p.channels);
}

// ---- second launch: the chunks' sums added, the group means made ---------------------------------------------------------------
// Workgroup (n, tile): join_cols channels (whole groups), 1 << fold_log2 lanes per channel.
template <typename T>
__global__ void __launch_bounds__(256) k_gn_bwd_join(const float* chunks, const T* gamma, float* sums, float* means, const GnShape p) {
  extern __shared__ __align__(16) float lds[];   // [2][join_cols], weighted by gamma
  const uint32_t tiles = (p.channels + p.join_cols - 1u) / p.join_cols;
  const uint32_t n = blockIdx.x / tiles, c0 = (blockIdx.x - n * tiles) * p.join_cols, c1 = min(c0 + p.join_cols, p.channels);
  const uint32_t lanes = 1u << p.fold_log2, at_once = 256u >> p.fold_log2;   // neighbouring threads: neighbouring channels
  const uint32_t lane = threadIdx.x / at_once, own = threadIdx.x - lane * at_once;
  __shared__ float part[2][256];
  const float* const from = chunks + (size_t)n * p.chunks * 2u * p.channels;
  const uint32_t pitch = p.sum_pitch;
  for (uint32_t cb = c0; cb < c1; cb += at_once) {
    const uint32_t c = min(cb + own, c1 - 1u);
    float a = 0.0f, b = 0.0f;
#pragma unroll 8
    for (uint32_t k = lane; k < p.chunks; k += lanes) {
      a += from[(size_t)k * 2u * p.channels + c];
      b += from[((size_t)k * 2u + 1u) * p.channels + c];
    }
    part[0][threadIdx.x] = a;
    part[1][threadIdx.x] = b;
    __syncthreads();
    if (lane == 0 && cb + own < c1) {
      for (uint32_t k = 1; k < lanes; ++k) {
        a += part[0][k * at_once + own];
        b += part[1][k * at_once + own];
      }
      float* const out = sums + (size_t)n * 2u * pitch + c;
      out[0] = a;
      out[pitch] = b;
      const float w = load1(gamma + c);
      lds[c - c0] = w * a;
      lds[p.join_cols + c - c0] = w * b;
    }
    __syncthreads();
  }
  const uint32_t groups = (c1 - c0) / p.dim;
  for (uint32_t g0 = 0; g0 < groups; g0 += 4u) {   // a wavefront per group
    const uint32_t g = g0 + (threadIdx.x >> 6), gc = min(g, groups - 1u);
    float m1 = 0.0f, m2 = 0.0f;
    for (uint32_t d = threadIdx.x & 63u; d < p.dim; d += 64u) {
      m1 += lds[gc * p.dim + d];
      m2 += lds[p.join_cols + gc * p.dim + d];
    }
    m1 = group_allreduce<OpSum>(m1, 64);
    m2 = group_allreduce<OpSum>(m2, 64);
    if ((threadIdx.x & 63u) == 0 && g < groups)
      *reinterpret_cast<f32x2*>(means + 2u * ((size_t)n * p.groups + c0 / p.dim + g)) = f32x2{m1 * p.inv_count, m2 * p.inv_count};
  }
}

// ---- third launch ------------------------------------------------------------------------------------------------------
template <typename T, int VEC, int ACT, bool FROM8>
__global__ void __launch_bounds__(256) k_gn_bwd_apply(const typename GnValue<T, FROM8>::type* x, const float* centre, const float* rstd, const T* gamma,
                                                      const T* beta, const T* dy, T* dx, const float* means, const GnShape p) {
  typedef typename GnValue<T, FROM8>::type X;
  constexpr int U = 4;
  const uint32_t width = p.set_groups * p.dim;
  const uint32_t bc = fast_div(blockIdx.x, p.div_sets), set = blockIdx.x - bc * p.sets;
  const uint32_t n = fast_div(bc, p.div_chunks), chunk = bc - n * p.chunks;
  const uint32_t r0 = chunk * p.chunk_rows, r1 = min(r0 + p.chunk_rows, p.positions);
  const GnLane l = gn_lane<VEC>(p);
  if (!l.live) return;
  const size_t base = (size_t)n * p.positions * p.channels + set * width + l.col;
  const uint32_t step = p.rows_at_once;
  uint32_t row = r0 + l.row;
  typename VecIo<X, VEC>::Raw nx[U], x0[U];
  typename VecIo<T, VEC>::Raw nd[U], d0[U];
  auto issue = [&]() {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const size_t at = base + min(row + u * step, r1 - 1u) * p.channels;
      nx[u] = VecIo<X, VEC>::template load<true>(x + at);
      nd[u] = VecIo<T, VEC>::template load<true>(dy + at);
    }
  };
  issue();
  GnChannels<T, VEC, FROM8> ch;
  ch.load(p, l, n, set, centre, rstd, gamma, beta);
  float m1[VEC], m2[VEC], r[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    const uint32_t g = n * p.groups + set * p.set_groups + fast_div(l.col + e, p.div_dim);
    const f32x2 m = *reinterpret_cast<const f32x2*>(means + 2u * (size_t)g);
    m1[e] = m.x;
    m2[e] = m.y;
    r[e] = FROM8 ? rstd[g] : ch.scale[e];
  }
  auto put = [&](typename VecIo<X, VEC>::Raw rx, typename VecIo<T, VEC>::Raw rd, uint32_t at) {
    float v[VEC], d[VEC];
    VecIo<X, VEC>::widen(rx, v);
    VecIo<T, VEC>::widen(rd, d);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float xh = ch.normal(v[e], e);
      const float dz = ch.template dz<ACT>(xh, d[e], e);
      d[e] = (__builtin_fmaf(dz, ch.ga[e], -m1[e]) - xh * m2[e]) * r[e];
    }
    VecIo<T, VEC>::store(dx + base + at * p.channels, d);
  };
  for (uint32_t all = r0 + U * step; all <= r1; all += U * step) {   // (every thread has the positions below `all`)
    const uint32_t at = row;
#pragma unroll
    for (int u = 0; u < U; ++u) x0[u] = nx[u], d0[u] = nd[u];
    row += U * step;
    issue();
#pragma unroll
    for (int u = 0; u < U; ++u) put(x0[u], d0[u], at + u * step);
  }
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (row + u * step < r1) put(nx[u], nd[u], row + u * step);
}

}  // namespace fsk

namespace fs {
using namespace fsk;

namespace {
template <typename T, int VEC, int ACT, bool FROM8>
const void* bwd_sym(int32_t kernel, const GroupNormP& p) {
  if (kernel == K_GN_BWD_SUMS) return (const void*)k_gn_bwd_sums<T, VEC, ACT, FROM8>;
  if (kernel == K_GN_BWD_APPLY) return (const void*)k_gn_bwd_apply<T, VEC, ACT, FROM8>;
  if (p.threads == 256) {
    switch (p.vecs_per_lane) {
      case 1: return (const void*)k_gn_bwd_slab<T, VEC, 1, ACT, FROM8, 256>;
      case 2: return (const void*)k_gn_bwd_slab<T, VEC, 2, ACT, FROM8, 256>;
      case 4: return (const void*)k_gn_bwd_slab<T, VEC, 4, ACT, FROM8, 256>;
    }
  } else if (p.threads == 512) {
    switch (p.vecs_per_lane) {
      case 4: return (const void*)k_gn_bwd_slab<T, VEC, 4, ACT, FROM8, 512>;
      case 8: return (const void*)k_gn_bwd_slab<T, VEC, 8, ACT, FROM8, 512>;
      case 16: return (const void*)k_gn_bwd_slab<T, VEC, 16, ACT, FROM8, 512>;
    }
  }
  return nullptr;
}
template <typename T, int VEC, int ACT>
const void* from_sym(int32_t kernel, const GroupNormP& p) {
  return p.checkpoint ? bwd_sym<T, VEC, ACT, true>(kernel, p) : bwd_sym<T, VEC, ACT, false>(kernel, p);
}
template <typename T, int VEC>
const void* bwd_act_sym(int32_t kernel, const GroupNormP& p) {
  switch (p.act) {
    case ACT_NONE: return from_sym<T, VEC, ACT_NONE>(kernel, p);
    case ACT_GELU: return from_sym<T, VEC, ACT_GELU>(kernel, p);
    case ACT_SILU: return from_sym<T, VEC, ACT_SILU>(kernel, p);
    default: return nullptr;
  }
}
template <typename T>
const void* bwd_type_sym(int32_t kernel, const GroupNormP& p) {
  if (kernel == K_GN_BWD_JOIN) return (const void*)k_gn_bwd_join<T>;
  return p.vec == 1 ? bwd_act_sym<T, 1>(kernel, p) : bwd_act_sym<T, Elem<T>::VEC>(kernel, p);
}
}  // namespace

const void* group_norm_backward_kernel_symbol(int32_t kernel, const KernelArgs& a) {
  const GroupNormP& p = a.u.gn;
  switch (p.dt) {
    case DT_F32: return bwd_type_sym<float>(kernel, p);
    case DT_F16: return bwd_type_sym<f16_t>(kernel, p);
    case DT_BF16: return bwd_type_sym<bf16_t>(kernel, p);
    default: return nullptr;
  }
}

}  // namespace fs
