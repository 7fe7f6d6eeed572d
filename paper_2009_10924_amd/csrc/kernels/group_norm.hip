// Group normalisation with an activation:  z = (x - mean) rstd gamma + beta,  y = act(z), mean and variance over the positions
// and channels of a group; beside it the 8-bit checkpoint of (x - mean) rstd.
//
// A group's values are read once where a workgroup can hold them (k_gn_slab).  Otherwise a first launch gathers mean and
// sum of squared deviations per chunk of positions, and a last one, which joins the chunks of its groups, reads x again; where
// that joins too many for every workgroup, a launch in between does it once.  Bound by memory from some 30 MB on: bf16
// [16, 16384, 256] with SiLU, 64 us for its 268 MB (24 us gather, 40 read and write again: 5.6 and 6.7 TB/s); smaller ones by what a
// workgroup does one after the other: bf16 [8, 4096, 320] with a checkpoint 19.4 us, 8.5 for its bytes alone.  No variance is a
// difference of large sums: inside registers it is the mean of squared deviations from the known mean, and partial results
// join as M2 = M2a + M2b + (mean_b - mean_a)^2 na nb / (na + nb).
#include <hip/hip_runtime.h>

#include "group_norm.hpp"
#include "kernel_table.hpp"

namespace fsk {
using namespace fs;

// ---- one launch: the set's values stay in registers ----------------------------------------------------------------------
template <typename T, int VEC, int K, bool WHOLE, int ACT, int NT>
__global__ void __launch_bounds__(NT) k_gn_slab(const T* x, const T* gamma, const T* beta, T* y, float* mean_out, float* rstd_out, e4m3_t* q,
                                                float* scale_out, const GnShape p) {
  extern __shared__ __align__(16) float lds[];
  constexpr int G = WHOLE ? 1 : VEC;   // groups that a vector can touch
  constexpr int ITEMS = WHOLE ? GN_ONE : GN_DENSE;
  const uint32_t width = p.set_groups * p.dim;
  const uint32_t n_items = p.rows_at_once * gn_pitch<ITEMS, VEC>(p);
  float* const items = lds;
  float* const most = lds + n_items;                       // with a checkpoint only
  float* const stat = lds + (q ? 2u : 1u) * n_items;       // [3][set_groups]
  const uint32_t b = gn_block(p.batch * p.sets), n = fast_div(b, p.div_sets), set = b - n * p.sets;
  const GnLane l = gn_lane<VEC>(p);
  const size_t base = (size_t)n * p.positions * p.channels + set * width;

  const uint32_t place = l.row * p.channels + l.col, step = p.rows_at_once * p.channels, last = (p.positions - 1u) * p.channels + l.col;

  typename VecIo<T, VEC>::Raw raw[K];
#pragma unroll
  for (int k = 0; k < K; ++k) raw[k] = VecIo<T, VEC>::template load<false>(near_element(x + base, min(place + (uint32_t)k * step, last)));
  GnParams<T, VEC> gains, shifts;
  gains.load(gamma, set * width + l.col, p.wide_params);
  shifts.load(beta, set * width + l.col, p.wide_params);

  auto valid = [&](int k) { return l.live && place + (uint32_t)k * step <= last; };
  float a[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) a[e] = 0.0f;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    float v[VEC];
    again(raw[k]);
    VecIo<T, VEC>::widen(raw[k], v);
#pragma unroll
    for (int e = 0; e < VEC; ++e) a[e] += valid(k) ? v[e] : 0.0f;
    done(a);
  }
  gn_deposit<ITEMS, VEC>(items, p, l, a);
  __syncthreads();
  gn_groups<ITEMS, VEC>(p, [&](uint32_t g, uint32_t lane, bool writes, uint32_t first, uint32_t per) {
    const float s = gn_fold<ITEMS, VEC, OpSum>(items, p, lane, first, per);
    if (writes) stat[g] = s * p.inv_count;
  });
  __syncthreads();
  uint32_t group[G];
  float mean[G];
#pragma unroll
  for (int i = 0; i < G; ++i) {
    group[i] = fast_div(l.col + i, p.div_dim);
    mean[i] = stat[group[i]];
  }
  float far[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) a[e] = far[e] = 0.0f;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    float v[VEC];
    again(raw[k]);
    VecIo<T, VEC>::widen(raw[k], v);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float c = valid(k) ? v[e] - mean[WHOLE ? 0 : e] : 0.0f;
      a[e] = __builtin_fmaf(c, c, a[e]);
      far[e] = fmaxf(far[e], __builtin_fabsf(c));
    }
    done(a);
    done(far);
  }
  gn_deposit<ITEMS, VEC>(items, p, l, a);
  if (q) gn_deposit_max<ITEMS, VEC>(most, p, l, far);
  __syncthreads();
  gn_groups<ITEMS, VEC>(p, [&](uint32_t g, uint32_t lane, bool writes, uint32_t first, uint32_t per) {
    const float r = fast_rsqrt(gn_fold<ITEMS, VEC, OpSum>(items, p, lane, first, per) * p.inv_count + p.eps);
    const float s = q ? scale_of(gn_fold<ITEMS, VEC, OpMax>(most, p, lane, first, per) * r, p.inv_max, p.tiny) : 0.0f;
    if (writes) {
      stat[p.set_groups + g] = r;
      stat[2u * p.set_groups + g] = s;
      const uint32_t at = n * p.groups + set * p.set_groups + g;
      if (mean_out) mean_out[at] = stat[g];
      if (rstd_out) rstd_out[at] = r;
      if (q) scale_out[at] = s;
    }
  });
  __syncthreads();
  float rstd[G], ga[VEC], be[VEC];
#pragma unroll
  for (int i = 0; i < G; ++i) rstd[i] = stat[p.set_groups + group[i]];
  gains.widen(p.wide_params, ga);
  shifts.widen(p.wide_params, be);
#pragma unroll
  for (int e = 0; e < VEC; ++e) ga[e] *= rstd[WHOLE ? 0 : e];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    again(raw[k]);
    if (!valid(k)) continue;
    float v[VEC];
    VecIo<T, VEC>::widen(raw[k], v);
#pragma unroll
    for (int e = 0; e < VEC; ++e)
      v[e] = activate<ACT>(__builtin_fmaf(v[e] - mean[WHOLE ? 0 : e], ga[e], be[e]));
    store_as<VecIo<T, VEC>>(p.whole_lines, near_element(y + base, place + (uint32_t)k * step), v);
  }
  if (!q) return;
  float to8[G];
#pragma unroll
  for (int i = 0; i < G; ++i) to8[i] = rstd[i] * Divisor(stat[2u * p.set_groups + group[i]]).inv;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    again(raw[k]);
    if (!valid(k)) continue;
    float v[VEC];
    VecIo<T, VEC>::widen(raw[k], v);
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = (v[e] - mean[WHOLE ? 0 : e]) * to8[WHOLE ? 0 : e];
    store_as<VecIo<e4m3_t, VEC>>(p.whole_lines, near_element(q + base, place + (uint32_t)k * step), v);
  }
}

// ---- first launch of several: statistics of a chunk of positions -----------------------------------------------------------
// out[batch][chunk][group] = mean, sum of squared deviations from it; behind all of them, for the scale of a checkpoint, lowest and
// highest value.  A thread adds up, for each of its channels, deviations from the mean c of its first four values and their
// squares: 4 operations per element where joining four by four took 8 (the launch is as much bound by its arithmetic as by
// memory: bf16 [8, 4096, 320] 9.8 us then).  M2 = sum d^2 - (sum d)^2 / n cancels no more than the thread's number of
// positions allows: the first four alone give M2 >= 4 (c - mean)^2, so what is taken off is at most n / 4 times what remains,
// and n is at most kGnMostRows.
template <typename T, int VEC, bool WHOLE, bool RANGE>
__global__ void __launch_bounds__(256) k_gn_stats(const T* x, float* out, const GnShape p) {
  extern __shared__ __align__(16) float lds[];
  constexpr int U = 4, ITEMS = WHOLE ? GN_ONE : RANGE ? GN_SPACED : GN_DENSE;
  const uint32_t width = p.set_groups * p.dim;
  const uint32_t n_items = p.rows_at_once * gn_pitch<ITEMS, VEC>(p);
  float* const means = lds;
  float* const squares = lds + n_items;
  float* const weight = lds + (RANGE ? 4u : 2u) * n_items;   // [rows_at_once]
  const uint32_t bc = fast_div(blockIdx.x, p.div_sets), set = blockIdx.x - bc * p.sets;
  const uint32_t n = fast_div(bc, p.div_chunks), chunk = bc - n * p.chunks;
  const uint32_t r0 = chunk * p.chunk_rows, r1 = min(r0 + p.chunk_rows, p.positions);
  const GnLane l = gn_lane<VEC>(p);
  const T* const from = x + (size_t)n * p.positions * p.channels + set * width + l.col;
  auto load = [&](uint32_t row) { return VecIo<T, VEC>::template load<false>(from + min(row, r1 - 1u) * p.channels); };

  float c[VEC], s1[VEC], s2[VEC], lo[VEC], hi[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) c[e] = s1[e] = s2[e] = 0.0f, lo[e] = __builtin_inff(), hi[e] = -__builtin_inff();
  const uint32_t step = p.rows_at_once, here = r1 - r0;
  const uint32_t mine = l.live && l.row < here ? (here - 1u - l.row) / step + 1u : 0u;   // this thread's positions
  if (l.live) {
    uint32_t row = r0 + l.row;
    typename VecIo<T, VEC>::Raw next[U], now[U];
#pragma unroll
    for (int u = 0; u < U; ++u) next[u] = load(row + u * step);
    // (positions behind the chunk's end repeat its last one; a centre may be any value of about the right size)
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float v[VEC];
      VecIo<T, VEC>::widen(next[u], v);
#pragma unroll
      for (int e = 0; e < VEC; ++e) c[e] = u == 0 ? v[e] : c[e] + v[e];
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) c[e] *= 1.0f / U;
    auto add = [&](typename VecIo<T, VEC>::Raw raw) {
      float v[VEC];
      VecIo<T, VEC>::widen(raw, v);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float d = v[e] - c[e];
        s1[e] += d;
        s2[e] = __builtin_fmaf(d, d, s2[e]);
        if constexpr (RANGE) lo[e] = fminf(lo[e], d), hi[e] = fmaxf(hi[e], d);
      }
    };
    auto add_two = [&](typename VecIo<T, VEC>::Raw raw, typename VecIo<T, VEC>::Raw other) {   // (a maximum of three is one operation)
      float v[VEC], w[VEC];
      VecIo<T, VEC>::widen(raw, v);
      VecIo<T, VEC>::widen(other, w);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float d = v[e] - c[e], f = w[e] - c[e];
        s1[e] += d;
        s2[e] = __builtin_fmaf(d, d, s2[e]);
        s1[e] += f;
        s2[e] = __builtin_fmaf(f, f, s2[e]);
        if constexpr (RANGE) lo[e] = fminf(fminf(lo[e], d), f), hi[e] = fmaxf(fmaxf(hi[e], d), f);
      }
    };
    for (uint32_t all = r0 + U * step; all <= r1; all += U * step) {   // (every live thread has the positions below `all`)
#pragma unroll
      for (int u = 0; u < U; ++u) now[u] = next[u];
      row += U * step;
#pragma unroll
      for (int u = 0; u < U; ++u) next[u] = load(row + u * step);
#pragma unroll
      for (int u = 0; u < U; u += 2) add_two(now[u], now[u + 1]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (row + u * step < r1) add(next[u]);
  }
  const float count = (float)mine, inv_mine = mine ? 1.0f / count : 0.0f;
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    const float m = s1[e] * inv_mine;
    if constexpr (RANGE) lo[e] += c[e], hi[e] += c[e];
    c[e] += m;
    s2[e] = fmaxf(__builtin_fmaf(-m, s1[e], s2[e]), 0.0f);
  }
  // the thread's channels of one group as one item: equal counts, so their mean is the mean of the means
  if constexpr (WHOLE) {
    float m = 0.0f, d = 0.0f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) m += c[e];
    m *= 1.0f / VEC;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float apart = c[e] - m;
      d += __builtin_fmaf(apart * apart, count, s2[e]);
      if constexpr (RANGE) lo[0] = fminf(lo[0], lo[e]), hi[0] = fmaxf(hi[0], hi[e]);
    }
    if (l.live) {
      const uint32_t at = l.row * p.set_vecs + l.vec;
      means[at] = m;
      squares[at] = d;
      if constexpr (RANGE) lds[2u * n_items + at] = lo[0], lds[3u * n_items + at] = hi[0];
    }
  } else {
    gn_deposit<ITEMS, VEC>(means, p, l, c);
    gn_deposit<ITEMS, VEC>(squares, p, l, s2);
    if constexpr (RANGE) {
      gn_deposit<ITEMS, VEC>(lds + 2u * n_items, p, l, lo);
      gn_deposit<ITEMS, VEC>(lds + 3u * n_items, p, l, hi);
    }
  }
  if (l.live && l.vec == 0) weight[l.row] = WHOLE ? count * VEC : count;
  __syncthreads();
  const float inv = 1.0f / ((float)here * (float)p.dim);
  gn_groups<ITEMS, VEC>(p, [&](uint32_t g, uint32_t lane, bool writes, uint32_t first, uint32_t per) {
    const uint32_t n_it = p.rows_at_once * per, lanes = 1u << p.fold_log2;
    float m = 0.0f, d = 0.0f, low = __builtin_inff(), high = -__builtin_inff();
#pragma unroll 4
    for (uint32_t i = lane; i < n_it; i += lanes) {
      const uint32_t rr = fast_div(i, p.div_per), at = rr * gn_pitch<ITEMS, VEC>(p) + gn_item<ITEMS, VEC>(first + (i - rr * per));
      m = __builtin_fmaf(weight[rr], means[at], m);
      if constexpr (RANGE) low = fminf(low, lds[2u * n_items + at]), high = fmaxf(high, lds[3u * n_items + at]);
    }
    m = group_allreduce<OpSum>(m, (int)lanes) * inv;
#pragma unroll 4
    for (uint32_t i = lane; i < n_it; i += lanes) {
      const uint32_t rr = fast_div(i, p.div_per), at = rr * gn_pitch<ITEMS, VEC>(p) + gn_item<ITEMS, VEC>(first + (i - rr * per));
      const float apart = means[at] - m;
      d += __builtin_fmaf(apart * apart, weight[rr], squares[at]);
    }
    d = group_allreduce<OpSum>(d, (int)lanes);
    if constexpr (RANGE) {
      high = group_allreduce<OpMax>(high, (int)lanes);
      low = -group_allreduce<OpMax>(-low, (int)lanes);
    }
    if (writes) {
      const size_t at = (size_t)bc * p.groups + set * p.set_groups + g;
      reinterpret_cast<f32x2*>(out)[at] = f32x2{m, d};
      if constexpr (RANGE) reinterpret_cast<f32x2*>(out)[(size_t)p.batch * p.chunks * p.groups + at] = f32x2{low, high};
    }
  });
}

// The chunks of a batch entry and group joined by `lanes` lanes: mean, rstd, scale of the checkpoint.  Called by whole
// wavefronts.  What it costs is the latency of its loads, so 16 per lane are under way together (four at a time, and once more
// for the deviations, made the last launch of bf16 [8, 4096, 320] with 86 chunks 7 us longer).
template <bool RANGE>
__device__ __forceinline__ void gn_join(const float* chunks, uint32_t n, uint32_t group, uint32_t lane, uint32_t lanes, const GnShape& p, float& mean,
                                        float& r, float& s) {
  constexpr int B = RANGE ? 8 : 16;
  const f32x2* const from = reinterpret_cast<const f32x2*>(chunks) + (size_t)n * p.chunks * p.groups + group;
  const f32x2* const range = from + (size_t)p.batch * p.chunks * p.groups;
  const float full = (float)p.chunk_rows * (float)p.dim;
  const float last = (float)(p.positions - (p.chunks - 1u) * p.chunk_rows) * (float)p.dim;
  float have = 0.0f, d = 0.0f, low = __builtin_inff(), high = -__builtin_inff();
  mean = 0.0f;
  for (uint32_t c0 = lane; c0 - lane < p.chunks; c0 += B * lanes) {
    f32x2 v[B], w[B];
#pragma unroll
    for (int i = 0; i < B; ++i) {
      const size_t at = (size_t)min(c0 + i * lanes, p.chunks - 1u) * p.groups;
      v[i] = from[at];
      if constexpr (RANGE) w[i] = range[at];
    }
    float m = 0.0f, dd = 0.0f, sum = 0.0f, weight[B];
#pragma unroll
    for (int i = 0; i < B; ++i) {
      const uint32_t c = c0 + i * lanes;
      weight[i] = c + 1u < p.chunks ? full : c + 1u == p.chunks ? last : 0.0f;
      sum += weight[i];
      m = __builtin_fmaf(weight[i], v[i].x, m);
      if constexpr (RANGE) low = fminf(low, w[i].x), high = fmaxf(high, w[i].y);
    }
    sum = group_allreduce<OpSum>(sum, (int)lanes);
    m = group_allreduce<OpSum>(m, (int)lanes) / sum;
#pragma unroll
    for (int i = 0; i < B; ++i) {
      const float apart = v[i].x - m;
      if (weight[i] > 0.0f) dd += __builtin_fmaf(apart * apart, weight[i], v[i].y);
    }
    dd = group_allreduce<OpSum>(dd, (int)lanes);
    const float all = have + sum, share = sum / all, apart = m - mean;
    mean = have > 0.0f ? __builtin_fmaf(apart, share, mean) : m;
    d += have > 0.0f ? __builtin_fmaf(apart * apart, have * share, dd) : dd;
    have = all;
  }
  r = fast_rsqrt(d * p.inv_count + p.eps);
  s = 0.0f;
  if constexpr (RANGE) {
    high = group_allreduce<OpMax>(high, (int)lanes);
    low = -group_allreduce<OpMax>(-low, (int)lanes);
    s = scale_of(fmaxf(high - mean, mean - low) * r, p.inv_max, p.tiny);
  }
}

// ---- a launch of its own for that, where every workgroup of the last launch would join too many chunks -----------------------
template <bool RANGE>
__global__ void __launch_bounds__(256) k_gn_join(const float* chunks, float* joined, float* mean_out, float* rstd_out, float* scale_out,
                                                 const GnShape p) {
  const uint32_t lanes = 1u << p.fold_log2, lane = threadIdx.x & (lanes - 1u);
  const uint32_t own = blockIdx.x * (256u >> p.fold_log2) + (threadIdx.x >> p.fold_log2);
  const uint32_t at = min(own, p.batch * p.groups - 1u), n = at / p.groups, g = at - n * p.groups;
  float m, r, s;
  gn_join<RANGE>(chunks, n, g, lane, lanes, p, m, r, s);
  if (lane != 0 || own >= p.batch * p.groups) return;
  *reinterpret_cast<f32x4*>(joined + (size_t)at * 4u) = f32x4{m, r, s, 0.0f};
  if (mean_out) mean_out[at] = m;
  if (rstd_out) rstd_out[at] = r;
  if (scale_out) scale_out[at] = s;
}

// ---- last launch -------------------------------------------------------------------------------------------------------
// JOIN: `stats` are the chunks', which every workgroup joins for its groups (the first one of a batch entry hands them out);
// otherwise they are joined already.
template <typename T, int VEC, bool WHOLE, int ACT, bool STORE8, bool JOIN>
__global__ void __launch_bounds__(256) k_gn_apply(const T* x, const T* gamma, const T* beta, const float* stats, T* y, e4m3_t* q, float* mean_out,
                                                  float* rstd_out, float* scale_out, const GnShape p) {
  extern __shared__ __align__(16) float lds[];   // JOIN: [set_groups][4]
  constexpr int U = 4, G = WHOLE ? 1 : VEC;
  const uint32_t width = p.set_groups * p.dim;
  const uint32_t bc = fast_div(blockIdx.x, p.div_sets), set = blockIdx.x - bc * p.sets;   // (the die that read it for k_gn_stats)
  const uint32_t n = fast_div(bc, p.div_chunks), chunk = bc - n * p.chunks;
  const uint32_t r0 = chunk * p.chunk_rows, r1 = min(r0 + p.chunk_rows, p.positions);
  const GnLane l = gn_lane<VEC>(p);
  const size_t base = (size_t)n * p.positions * p.channels + set * width + l.col;
  auto load = [&](uint32_t row) { return VecIo<T, VEC>::template load<true>(x + base + min(row, r1 - 1u) * p.channels); };
  const uint32_t step = p.rows_at_once;
  uint32_t row = r0 + l.row;
  typename VecIo<T, VEC>::Raw next[U], now[U];
#pragma unroll
  for (int u = 0; u < U; ++u) next[u] = load(row + u * step);
  GnParams<T, VEC> gains, shifts;
  gains.load(gamma, set * width + l.col, p.wide_params);
  shifts.load(beta, set * width + l.col, p.wide_params);
  if constexpr (JOIN) {
    const uint32_t lanes = 1u << p.fold_log2, sets = 256u >> p.fold_log2, lane = threadIdx.x & (lanes - 1u);
    for (uint32_t g0 = 0; g0 < p.set_groups; g0 += sets) {
      const uint32_t g = g0 + (threadIdx.x >> p.fold_log2), at = set * p.set_groups + min(g, p.set_groups - 1u);
      float m, r, s;
      gn_join<STORE8>(stats, n, at, lane, lanes, p, m, r, s);
      if (lane == 0 && g < p.set_groups) {
        *reinterpret_cast<f32x4*>(lds + 4u * g) = f32x4{m, r, s, 0.0f};
        if (chunk == 0) {
          if (mean_out) mean_out[n * p.groups + at] = m;
          if (rstd_out) rstd_out[n * p.groups + at] = r;
          if (scale_out) scale_out[n * p.groups + at] = s;
        }
      }
    }
    __syncthreads();
  }
  if (!l.live) return;
  float mean[G], rstd[G], to8[G];
#pragma unroll
  for (int i = 0; i < G; ++i) {
    const uint32_t g = fast_div(l.col + i, p.div_dim);
    const f32x4 j = *reinterpret_cast<const f32x4*>(JOIN ? lds + 4u * g : stats + (size_t)(n * p.groups + set * p.set_groups + g) * 4u);
    mean[i] = j.x;
    rstd[i] = j.y;
    if constexpr (STORE8) to8[i] = j.y * Divisor(j.z).inv;
  }
  float ga[VEC], be[VEC];
  gains.widen(p.wide_params, ga);
  shifts.widen(p.wide_params, be);
#pragma unroll
  for (int e = 0; e < VEC; ++e) ga[e] *= rstd[WHOLE ? 0 : e];
  auto put = [&](typename VecIo<T, VEC>::Raw raw, uint32_t at) {
    float v[VEC], z[VEC];
    VecIo<T, VEC>::widen(raw, v);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      v[e] -= mean[WHOLE ? 0 : e];
      z[e] = activate<ACT>(__builtin_fmaf(v[e], ga[e], be[e]));
    }
    VecIo<T, VEC>::store(y + base + at * p.channels, z);
    if constexpr (STORE8) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[e] *= to8[WHOLE ? 0 : e];
      VecIo<e4m3_t, VEC>::store(q + base + at * p.channels, v);
    }
  };
  for (uint32_t all = r0 + U * step; all <= r1; all += U * step) {   // (every thread has the positions below `all`)
    const uint32_t at = row;
#pragma unroll
    for (int u = 0; u < U; ++u) now[u] = next[u];
    row += U * step;
#pragma unroll
    for (int u = 0; u < U; ++u) next[u] = load(row + u * step);
#pragma unroll
    for (int u = 0; u < U; ++u) put(now[u], at + u * step);
  }
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (row + u * step < r1) put(next[u], row + u * step);
}

}  // namespace fsk

namespace fs {
using namespace fsk;

namespace {
template <typename T, int VEC, bool WHOLE, int ACT>
const void* slab_sym(const GroupNormP& p) {
  if (p.threads == 64) {
    switch (p.vecs_per_lane) {
      case 1: return (const void*)k_gn_slab<T, VEC, 1, WHOLE, ACT, 64>;
      case 2: return (const void*)k_gn_slab<T, VEC, 2, WHOLE, ACT, 64>;
      case 4: return (const void*)k_gn_slab<T, VEC, 4, WHOLE, ACT, 64>;
    }
  } else if (p.threads == 256) {
    switch (p.vecs_per_lane) {
      case 1: return (const void*)k_gn_slab<T, VEC, 1, WHOLE, ACT, 256>;
      case 2: return (const void*)k_gn_slab<T, VEC, 2, WHOLE, ACT, 256>;
      case 4: return (const void*)k_gn_slab<T, VEC, 4, WHOLE, ACT, 256>;
      case 8: return (const void*)k_gn_slab<T, VEC, 8, WHOLE, ACT, 256>;
    }
  } else if (p.threads == 512) {
    switch (p.vecs_per_lane) {
      case 4: return (const void*)k_gn_slab<T, VEC, 4, WHOLE, ACT, 512>;
      case 8: return (const void*)k_gn_slab<T, VEC, 8, WHOLE, ACT, 512>;
      case 16: return (const void*)k_gn_slab<T, VEC, 16, WHOLE, ACT, 512>;
      case 32: return (const void*)k_gn_slab<T, VEC, 32, WHOLE, ACT, 512>;
    }
  }
  return nullptr;
}
template <typename T, int VEC, bool WHOLE, int ACT>
const void* apply_sym(const GroupNormP& p) {
  if (p.checkpoint) return p.join ? (const void*)k_gn_apply<T, VEC, WHOLE, ACT, true, true> : (const void*)k_gn_apply<T, VEC, WHOLE, ACT, true, false>;
  return p.join ? (const void*)k_gn_apply<T, VEC, WHOLE, ACT, false, true> : (const void*)k_gn_apply<T, VEC, WHOLE, ACT, false, false>;
}
template <typename T, int VEC, bool WHOLE>
const void* act_sym(int32_t kernel, const GroupNormP& p) {
  if (kernel == K_GN_STATS) return p.checkpoint ? (const void*)k_gn_stats<T, VEC, WHOLE, true> : (const void*)k_gn_stats<T, VEC, WHOLE, false>;
  if (kernel == K_GN_SLAB) {
    switch (p.act) {
      case ACT_NONE: return slab_sym<T, VEC, WHOLE, ACT_NONE>(p);
      case ACT_GELU: return slab_sym<T, VEC, WHOLE, ACT_GELU>(p);
      case ACT_SILU: return slab_sym<T, VEC, WHOLE, ACT_SILU>(p);
      default: return nullptr;
    }
  }
  switch (p.act) {
    case ACT_NONE: return apply_sym<T, VEC, WHOLE, ACT_NONE>(p);
    case ACT_GELU: return apply_sym<T, VEC, WHOLE, ACT_GELU>(p);
    case ACT_SILU: return apply_sym<T, VEC, WHOLE, ACT_SILU>(p);
    default: return nullptr;
  }
}
template <typename T>
const void* type_sym(int32_t kernel, const GroupNormP& p) {
  if (p.vec == 1) return act_sym<T, 1, true>(kernel, p);
  return p.whole ? act_sym<T, Elem<T>::VEC, true>(kernel, p) : act_sym<T, Elem<T>::VEC, false>(kernel, p);
}
}  // namespace

const void* group_norm_kernel_symbol(int32_t kernel, const KernelArgs& a) {
  const GroupNormP& p = a.u.gn;
  if (kernel == K_GN_JOIN) return p.checkpoint ? (const void*)k_gn_join<true> : (const void*)k_gn_join<false>;
  switch (p.dt) {
    case DT_F32: return type_sym<float>(kernel, p);
    case DT_F16: return type_sym<f16_t>(kernel, p);
    case DT_BF16: return type_sym<bf16_t>(kernel, p);
    default: return nullptr;
  }
}

}  // namespace fs
