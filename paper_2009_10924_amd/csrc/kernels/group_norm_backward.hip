// Backward pass of group normalisation with an activation.  With xh the normalised values ((x - mean) rstd, or an 8-bit
// checkpoint times its scale), dz = dy act'(xh gamma + beta) and, per batch entry and channel,
//     A = sum over positions of dz,   B = sum over positions of dz xh
// everything else follows: dbeta = sum_n A, dgamma = sum_n B, and for a group's n values
//     m1 = sum_d gamma A / n,   m2 = sum_d gamma B / n,   dx = (gamma dz - m1 - xh m2) rstd.
// A workgroup that holds a set's values (k_gn_bwd_slab) reads them once, and K_COLFOLD adds up the batch; otherwise a first launch
// gathers A and B per chunk of positions and a second one, which adds up the chunks, reads the values again.
// Large calls are bound by memory and, with the GELU's slope, by arithmetic: f16 [8, 16384, 512] from x, 118 us for 403 MB (54 us
// gather at 5.0 TB/s, the vector units two thirds busy; 66 read and write at 6.2).  Smaller ones by what a workgroup does one after
// the other: bf16 [8, 4096, 320] from a checkpoint 23.4 us (11.9 + 12.3 as kernels), 8.5 for its bytes alone.
#include <hip/hip_runtime.h>

#include "fold.hpp"
#include "group_norm.hpp"
#include "kernel_table.hpp"

namespace fsk {
using namespace fs;

// The normalised values' storage: their 8-bit checkpoint, or the input.
template <typename T, bool FROM8> struct GnValue { typedef T type; };
template <typename T> struct GnValue<T, true> { typedef e4m3_t type; };

// What a thread knows of its channels.  Its values are worked on about their mean, v - shift (an 8-bit value as it is), and the
// factor that makes xh of them is multiplied into what is per channel: z = (v - shift) (scale gamma) + beta,  sum dz xh = scale
// sum dz (v - shift).  dx needs scale rstd, of values and their mean a square that is no float32 for deviations below 1e-19: then
// they are worked on times 2^50, exactly and at no cost (the subtraction is the end of a product), and scale is that much smaller.
template <typename T, int VEC, bool FROM8>
struct GnChannels {
  float shift[VEC], scale[VEC], slope[VEC], be[VEC], ga[VEC], times;
  // `centre`: means, or the checkpoint's scales
  __device__ __forceinline__ void load(const GnShape& p, const GnLane& l, uint32_t n, uint32_t set, const float* centre, const float* rstd,
                                       const T* gamma, const T* beta) {
    const uint32_t c = set * p.set_groups * p.dim + l.col, g0 = n * p.groups;
    GnParams<T, VEC> params;
    params.load(gamma, c, p.wide_params);
    params.widen(p.wide_params, ga);
    if (beta) {
      params.load(beta, c, p.wide_params);
      params.widen(p.wide_params, be);
    }
    // one group: one pair of values (as many loads as channels otherwise, which in the small shapes is what a thread mostly does)
    const uint32_t first = g0 + fast_div(c, p.div_dim);
    const float t0 = centre[first], r0 = FROM8 ? t0 : rstd[first];
#pragma unroll
    for (int e = 0; e < VEC; ++e) shift[e] = FROM8 ? 0.0f : t0, scale[e] = r0;
    if (!p.whole) {
#pragma unroll
      for (int e = 1; e < VEC; ++e) {
        const uint32_t g = g0 + fast_div(c + e, p.div_dim);
        shift[e] = FROM8 ? 0.0f : centre[g];
        scale[e] = FROM8 ? centre[g] : rstd[g];
      }
    }
    if constexpr (!FROM8) {
      float most = scale[0];
#pragma unroll
      for (int e = 1; e < VEC; ++e) most = fmaxf(most, scale[e]);
      const bool large = most > 0x1p50f;
      times = large ? 0x1p50f : 1.0f;
#pragma unroll
      for (int e = 0; e < VEC; ++e) shift[e] *= -times, scale[e] *= large ? 0x1p-50f : 1.0f;
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) slope[e] = scale[e] * ga[e];
  }
  __device__ __forceinline__ float about_mean(float v, int e) const { return FROM8 ? v : __builtin_fmaf(v, times, shift[e]); }
  __device__ __forceinline__ float rstd_of(int e) const { return scale[e] * times; }   // of values and their mean
  template <int ACT>
  __device__ __forceinline__ float dz(float v, float dy, int e) const {   // v: about its mean
    if constexpr (ACT == ACT_NONE) return dy;
    else return dy * activation_slope<ACT>(__builtin_fmaf(v, slope[e], be[e]));
  }
};
// dx = (gamma dz - m1 - xh m2) rstd = dz (gamma rstd) + ((v - shift) (-m2 scale rstd) - m1 rstd)
template <int VEC>
struct GnGradient {
  float by_dz[VEC], by_v[VEC], off[VEC];
  __device__ __forceinline__ float dx(float v, float dz, int e) const { return __builtin_fmaf(dz, by_dz[e], __builtin_fmaf(v, by_v[e], off[e])); }
  template <typename C>
  __device__ __forceinline__ void set(int e, const C& ch, float rstd, float m1, float m2) {
    by_dz[e] = ch.ga[e] * rstd;
    by_v[e] = -m2 * rstd * ch.scale[e];
    off[e] = -m1 * rstd;
  }
};

// Sums over the workgroup's positions of what every thread has gathered per channel, for channel c of the set to out_a[c] and
// out_b[c], and times gamma to weighted[c] and weighted[width + c], by 1 << fold_log2 lanes each.  Over several batch entries the sums
// go into `totals`, and with the last one to the outputs.  (Both in one go: two barriers and a chain of loads less than one after the
// other, 3 % of the calls with two launches and up to 20 % of those with many short entries.)
constexpr int kGnSums = GN_SPACED;
template <int VEC>
__device__ __forceinline__ void gn_channel_sums(float* items, const GnShape& p, const GnLane& l, const float (&a)[VEC], const float (&b)[VEC], const float* gain,
                                                float* weighted, float* out_a, float* out_b, float* totals = nullptr, bool first = true, bool last = true) {
  const uint32_t width = p.set_groups * p.dim, pitch = gn_pitch<kGnSums, VEC>(p), n_items = p.rows_at_once * pitch, lanes = 1u << p.fold_log2, lane = threadIdx.x & (lanes - 1u);
  gn_deposit<kGnSums, VEC>(items, p, l, a);
  gn_deposit<kGnSums, VEC>(items + n_items, p, l, b);
  __syncthreads();
  for (uint32_t c0 = 0; c0 < width; c0 += blockDim.x >> p.fold_log2) {
    const uint32_t c = c0 + (threadIdx.x >> p.fold_log2), cc = min(c, width - 1u), from = gn_item<kGnSums, VEC>(cc);
    float sa = 0.0f, sb = 0.0f;
#pragma unroll 4
    for (uint32_t r = lane; r < p.rows_at_once; r += lanes) {
      sa += items[from + r * pitch];
      sb += items[n_items + from + r * pitch];
    }
    sa = group_allreduce<OpSum>(sa, (int)lanes);
    sb = group_allreduce<OpSum>(sb, (int)lanes);
    if (lane == 0 && c < width) {
      weighted[c] = sa * gain[c];
      weighted[width + c] = sb * gain[c];
      if (!first) sa += totals[c], sb += totals[width + c];
      if (last) out_a[c] = sa, out_b[c] = sb;
      else totals[c] = sa, totals[width + c] = sb;
    }
  }
  __syncthreads();
}
// gamma of the set's channels in LDS (the first position's threads have them all)
template <int VEC>
__device__ __forceinline__ void gn_keep_gain(float* gain, const GnLane& l, const float (&ga)[VEC]) {
  if (l.row != 0) return;
#pragma unroll
  for (int e = 0; e < VEC; ++e) gain[l.col + e] = ga[e];
}
// A group's means m1 and m2 from its channels' weighted sums in LDS, 1 << means_log2 lanes per group: f(group, m1, m2) on the
// first of them.  (A wavefront per group, with gamma from memory, took 5 us of the 16 of f16 [2, 16384, 512].)
template <typename F>
__device__ __forceinline__ void gn_group_means(const GnShape& p, const float* wa, const float* wb, F&& f) {
  const uint32_t lanes = 1u << p.means_log2, lane = threadIdx.x & (lanes - 1u);
  for (uint32_t g0 = 0; g0 < p.set_groups; g0 += blockDim.x >> p.means_log2) {
    const uint32_t g = g0 + (threadIdx.x >> p.means_log2), gc = min(g, p.set_groups - 1u);
    float m1 = 0.0f, m2 = 0.0f;
#pragma unroll 4
    for (uint32_t d = lane; d < p.dim; d += lanes) {
      m1 += wa[gc * p.dim + d];
      m2 += wb[gc * p.dim + d];
    }
    m1 = group_allreduce<OpSum>(m1, (int)lanes);
    m2 = group_allreduce<OpSum>(m2, (int)lanes);
    if (lane == 0 && g < p.set_groups) f(g, m1 * p.inv_count, m2 * p.inv_count);
  }
}

// ---- one launch (and the fold, where more than one workgroup has a channel) ------------------------------------------------------
// A and B go to row n of out_a and out_b, rows 2 * sum_pitch floats apart (with one batch entry they are dbeta and dgamma).  MANY: a
// workgroup works through `entries` batch entries, one after the other, and adds up theirs, row i being the i-th workgroup's.
template <typename T, int VEC, int K, int ACT, bool FROM8, int NT, bool MANY>
__global__ void __launch_bounds__(NT) k_gn_bwd_slab(const typename GnValue<T, FROM8>::type* x, const float* centre, const float* rstd, const T* gamma,
                                                    const T* beta, const T* dy, T* dx, float* out_a, float* out_b, const GnShape p) {
  typedef typename GnValue<T, FROM8>::type X;
  extern __shared__ __align__(16) float lds[];
  const uint32_t width = p.set_groups * p.dim;
  float* const items = lds;
  float* const gain = lds + 2u * p.rows_at_once * gn_pitch<kGnSums, VEC>(p);
  float* const sum_a = gain + width;
  float* const sum_b = sum_a + width;
  float* const means = sum_b + width;   // [set_groups][2]
  float* const totals = means + 2u * p.set_groups;   // [2][width], for more than one entry
  const uint32_t b = gn_block(p.entry_blocks * p.sets), row = fast_div(b, p.div_sets), set = b - row * p.sets;
  const GnLane l = gn_lane<VEC>(p);
  const uint32_t n0 = MANY ? row * p.entries : row, n1 = MANY ? min(n0 + p.entries, p.batch) : n0 + 1u;
  const size_t out = (size_t)row * 2u * p.sum_pitch + set * width;
  for (uint32_t n = n0; n < n1; ++n) {
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
    gn_keep_gain<VEC>(gain, l, ch.ga);
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
        v[e] = ch.about_mean(v[e], e);
        const float dz = valid(k) ? ch.template dz<ACT>(v[e], d[e], e) : 0.0f;
        a[e] += dz;
        bb[e] = __builtin_fmaf(dz, valid(k) ? v[e] : 0.0f, bb[e]);
      }
      done(a);
      done(bb);
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) bb[e] *= ch.scale[e];
    gn_channel_sums<VEC>(items, p, l, a, bb, gain, sum_a, out_a + out, out_b + out, totals, !MANY || n == n0, !MANY || n + 1u == n1);
    gn_group_means(p, sum_a, sum_b, [&](uint32_t g, float m1, float m2) {
      means[2u * g] = m1;
      means[2u * g + 1u] = m2;
    });
    __syncthreads();
    GnGradient<VEC> gr;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const uint32_t g = fast_div(l.col + e, p.div_dim);
      gr.set(e, ch, FROM8 ? rstd[n * p.groups + set * p.set_groups + g] : ch.rstd_of(e), means[2u * g], means[2u * g + 1u]);
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
        v[e] = ch.about_mean(v[e], e);
        d[e] = gr.dx(v[e], ch.template dz<ACT>(v[e], d[e], e), e);
      }
      store_as<VecIo<T, VEC>>(p.whole_lines, near_element(dx + base, place + (uint32_t)k * step), d);
    }
  }
}

// ---- first launch of two: A and B of a chunk of positions, and what they add to the group means --------------------------------
// sums[batch][chunk][2][sum_pitch], means[batch][chunk][group][2]
template <typename T, int VEC, int ACT, bool FROM8>
__global__ void __launch_bounds__(256) k_gn_bwd_sums(const typename GnValue<T, FROM8>::type* x, const float* centre, const float* rstd, const T* gamma,
                                                     const T* beta, const T* dy, float* sums, float* means, const GnShape p) {
  typedef typename GnValue<T, FROM8>::type X;
  extern __shared__ __align__(16) float lds[];
  constexpr int U = 4;
  const uint32_t width = p.set_groups * p.dim;
  float* const gain = lds + 2u * p.rows_at_once * gn_pitch<kGnSums, VEC>(p);
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
    gn_keep_gain<VEC>(gain, l, ch.ga);
    auto add = [&](typename VecIo<X, VEC>::Raw rx, typename VecIo<T, VEC>::Raw rd) {
      float v[VEC], d[VEC];
      VecIo<X, VEC>::widen(rx, v);
      VecIo<T, VEC>::widen(rd, d);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        v[e] = ch.about_mean(v[e], e);
        const float dz = ch.template dz<ACT>(v[e], d[e], e);
        a[e] += dz;
        b[e] = __builtin_fmaf(dz, v[e], b[e]);
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
#pragma unroll
    for (int e = 0; e < VEC; ++e) b[e] *= ch.scale[e];
  }
  float* const to = sums + (size_t)bc * 2u * p.sum_pitch + set * width;
  float* const sum_a = gain + width;
  float* const sum_b = sum_a + width;
  gn_channel_sums<VEC>(lds, p, l, a, b, gain, sum_a, to, to + p.sum_pitch);
  float* const group_to = means + 2u * ((size_t)bc * p.groups + set * p.set_groups);
  gn_group_means(p, sum_a, sum_b,
                 [&](uint32_t g, float m1, float m2) { *reinterpret_cast<f32x2*>(group_to + 2u * g) = f32x2{m1, m2}; });
}

// ---- a launch between them, where every workgroup of the second one would add up too many chunks ---------------------------------
// joined[batch][group][2], 1 << fold_log2 lanes each
__device__ __forceinline__ f32x2 gn_bwd_join(const float* means, uint32_t n, uint32_t group, uint32_t lane, uint32_t lanes, const GnShape& p) {
  const f32x2* const from = reinterpret_cast<const f32x2*>(means) + (size_t)n * p.chunks * p.groups + group;
  constexpr int B = 16;   // loads that are under way together: their latency is what this costs
  float m1 = 0.0f, m2 = 0.0f;
  for (uint32_t c0 = lane; c0 - lane < p.chunks; c0 += B * lanes) {
    f32x2 v[B];
#pragma unroll
    for (int i = 0; i < B; ++i) v[i] = from[(size_t)min(c0 + i * lanes, p.chunks - 1u) * p.groups];
#pragma unroll
    for (int i = 0; i < B; ++i) {
      m1 += c0 + i * lanes < p.chunks ? v[i].x : 0.0f;
      m2 += c0 + i * lanes < p.chunks ? v[i].y : 0.0f;
    }
  }
  return f32x2{group_allreduce<OpSum>(m1, (int)lanes), group_allreduce<OpSum>(m2, (int)lanes)};
}
__global__ void __launch_bounds__(256) k_gn_bwd_join(const float* means, float* joined, const GnShape p) {
  const uint32_t lanes = 1u << p.fold_log2, lane = threadIdx.x & (lanes - 1u);
  const uint32_t own = blockIdx.x * (256u >> p.fold_log2) + (threadIdx.x >> p.fold_log2);
  const uint32_t at = min(own, p.batch * p.groups - 1u), n = at / p.groups;
  const f32x2 m = gn_bwd_join(means, n, at - n * p.groups, lane, lanes, p);
  if (lane == 0 && own < p.batch * p.groups) *reinterpret_cast<f32x2*>(joined + 2u * (size_t)at) = m;
}

// ---- second launch -----------------------------------------------------------------------------------------------------
// The first fold_blocks workgroups add up the chunks' A and B to dbeta and dgamma, beside the others.  JOIN: `means` are the
// chunks', which every workgroup adds up for its groups.
template <typename T, int VEC, int ACT, bool FROM8, bool JOIN>
__global__ void __launch_bounds__(256) k_gn_bwd_apply(const typename GnValue<T, FROM8>::type* x, const float* centre, const float* rstd, const T* gamma,
                                                      const T* beta, const T* dy, T* dx, const float* means, const float* sums, float* dbeta,
                                                      float* dgamma, const GnShape p) {
  typedef typename GnValue<T, FROM8>::type X;
  extern __shared__ __align__(16) float lds[];   // JOIN: [set_groups][2]; the fold's workgroups: 256 quads
  if (blockIdx.x < p.fold_blocks) {
    const uint32_t rows = p.batch * p.chunks, width = 2u * p.sum_pitch;
    f32x4* const quads = reinterpret_cast<f32x4*>(lds);
    if (rows > 128u) fold_tile<4, 64>(sums, dbeta, dgamma, rows, width, width, p.sum_pitch, p.channels, blockIdx.x, quads, kFoldF32);
    else fold_tile<16, 16>(sums, dbeta, dgamma, rows, width, width, p.sum_pitch, p.channels, blockIdx.x, quads, kFoldF32);
    return;
  }
  constexpr int U = 4;
  const uint32_t width = p.set_groups * p.dim;
  const uint32_t block = blockIdx.x - p.fold_blocks;   // (fold_blocks is a multiple of 8: on the die that read it for k_gn_bwd_sums)
  const uint32_t bc = fast_div(block, p.div_sets), set = block - bc * p.sets;
  const uint32_t n = fast_div(bc, p.div_chunks), chunk = bc - n * p.chunks;
  const uint32_t r0 = chunk * p.chunk_rows, r1 = min(r0 + p.chunk_rows, p.positions);
  const GnLane l = gn_lane<VEC>(p);
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
  if constexpr (JOIN) {
    const uint32_t lanes = 1u << p.fold_log2, sets = 256u >> p.fold_log2, lane = threadIdx.x & (lanes - 1u);
    for (uint32_t g0 = 0; g0 < p.set_groups; g0 += sets) {
      const uint32_t g = g0 + (threadIdx.x >> p.fold_log2);
      const f32x2 m = gn_bwd_join(means, n, set * p.set_groups + min(g, p.set_groups - 1u), lane, lanes, p);
      if (lane == 0 && g < p.set_groups) *reinterpret_cast<f32x2*>(lds + 2u * g) = m;
    }
    __syncthreads();
  }
  if (!l.live) return;
  GnGradient<VEC> gr;
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    const uint32_t g = fast_div(l.col + e, p.div_dim), at = n * p.groups + set * p.set_groups + g;
    const f32x2 m = *reinterpret_cast<const f32x2*>(JOIN ? lds + 2u * g : means + 2u * (size_t)at);
    gr.set(e, ch, FROM8 ? rstd[at] : ch.rstd_of(e), m.x, m.y);
  }
  auto put = [&](typename VecIo<X, VEC>::Raw rx, typename VecIo<T, VEC>::Raw rd, uint32_t at) {
    float v[VEC], d[VEC];
    VecIo<X, VEC>::widen(rx, v);
    VecIo<T, VEC>::widen(rd, d);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      v[e] = ch.about_mean(v[e], e);
      d[e] = gr.dx(v[e], ch.template dz<ACT>(v[e], d[e], e), e);
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
    for (int u = 0; u < U; ++u) {
      again(x0[u]);
      again(d0[u]);
      put(x0[u], d0[u], at + u * step);
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (row + u * step < r1) put(nx[u], nd[u], row + u * step);
}

}  // namespace fsk

namespace fs {
using namespace fsk;

namespace {
template <typename T, int VEC, int ACT, bool FROM8, int NT, bool MANY>
const void* slab_sym(int vecs) {
  switch (vecs) {
    case 1: return (const void*)k_gn_bwd_slab<T, VEC, 1, ACT, FROM8, NT, MANY>;
    case 2: return (const void*)k_gn_bwd_slab<T, VEC, 2, ACT, FROM8, NT, MANY>;
    case 4: return (const void*)k_gn_bwd_slab<T, VEC, 4, ACT, FROM8, NT, MANY>;
    default: return nullptr;
  }
}
template <typename T, int VEC, int ACT, bool FROM8>
const void* bwd_sym(int32_t kernel, const GroupNormP& p) {
  if (kernel == K_GN_BWD_SUMS) return (const void*)k_gn_bwd_sums<T, VEC, ACT, FROM8>;
  if (kernel == K_GN_BWD_APPLY)
    return p.join ? (const void*)k_gn_bwd_apply<T, VEC, ACT, FROM8, true> : (const void*)k_gn_bwd_apply<T, VEC, ACT, FROM8, false>;
  if (p.entries > 1) {   // batches of very many entries: workgroups of one wavefront or four
    if (p.threads == 64) return slab_sym<T, VEC, ACT, FROM8, 64, true>(p.vecs_per_lane);
    return p.threads == 256 ? slab_sym<T, VEC, ACT, FROM8, 256, true>(p.vecs_per_lane) : nullptr;
  }
  if (p.threads == 64) return slab_sym<T, VEC, ACT, FROM8, 64, false>(p.vecs_per_lane);
  if (p.threads == 256) return slab_sym<T, VEC, ACT, FROM8, 256, false>(p.vecs_per_lane);
  if (p.threads == 512) {
    switch (p.vecs_per_lane) {
      case 4: return (const void*)k_gn_bwd_slab<T, VEC, 4, ACT, FROM8, 512, false>;
      case 8: return (const void*)k_gn_bwd_slab<T, VEC, 8, ACT, FROM8, 512, false>;
      case 16: return (const void*)k_gn_bwd_slab<T, VEC, 16, ACT, FROM8, 512, false>;
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
  return p.vec == 1 ? bwd_act_sym<T, 1>(kernel, p) : bwd_act_sym<T, Elem<T>::VEC>(kernel, p);
}
}  // namespace

const void* group_norm_backward_kernel_symbol(int32_t kernel, const KernelArgs& a) {
  const GroupNormP& p = a.u.gn;
  if (kernel == K_GN_BWD_JOIN) return (const void*)k_gn_bwd_join;
  switch (p.dt) {
    case DT_F32: return bwd_type_sym<float>(kernel, p);
    case DT_F16: return bwd_type_sym<f16_t>(kernel, p);
    case DT_BF16: return bwd_type_sym<bf16_t>(kernel, p);
    default: return nullptr;
  }
}

}  // namespace fs
