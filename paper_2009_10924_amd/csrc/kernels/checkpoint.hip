// 8-bit activation checkpoints.
//   store:  z = x (+ bias),  s = max |z| over a block / 448 + tiny,  q = e4m3(z / s),  y = act(z) where there is one
//   use:    z = q s;  the values themselves, or dx = dy act'(z) and its column sums (the bias gradient)
// A block is a run of `cols` values (a row of the kernel's row space), so one lane group or workgroup holds it in registers
// between its maximum and its quotients: x is read once.  All are bound by memory (5.8 TB/s with bias, GELU and checkpoint of bf16
// [16384, 32 x 128], 58 us, the vector units 85 % busy; 7.1 restoring bf16 [8192, 64 x 128], 28.5 us, a part of it from the
// caches; 6.2 with GELU's slope and column sums, 57 us and the fold) but for small ones, which are a launch.
#include <hip/hip_runtime.h>

#include "activation.hpp"
#include "kernel_table.hpp"
#include "vec_access.hpp"

namespace fsk {
using namespace fs;

// ---- store -----------------------------------------------------------------------------------------------------------
// BLOCK: the whole workgroup on a row, otherwise 1 << lanes_log2 lanes; K vectors per lane.  The last vector of a row whose
// length is no multiple of VEC starts early, at the row's last VEC elements: the lane and its neighbour then write the same
// values to the elements that they share.
template <typename T, int VEC, int K, int ACT, bool BLOCK, bool STREAM>
__global__ void __launch_bounds__(BLOCK ? 1024 : 256) k_checkpoint(const T* x, const T* bias, T* y, e4m3_t* q, float* scale, uint32_t rows,
                                                                 uint32_t cols, int32_t lanes_log2, float inv_max, float tiny, uint32_t period_d,
                                                                 uint32_t period_m, uint32_t period_s) {
  __shared__ float slot[16];
  const uint32_t L = BLOCK ? blockDim.x : 1u << lanes_log2;
  const uint32_t lane = BLOCK ? threadIdx.x : threadIdx.x & (L - 1u);
  const uint32_t row = BLOCK ? blockIdx.x : blockIdx.x * (256u >> lanes_log2) + (threadIdx.x >> lanes_log2);
  const uint32_t r = min(row, rows - 1u);
  const size_t base = (size_t)r * cols;
  typename VecIo<T, VEC>::Raw rx[K], rb[K];
  uint32_t col[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    col[k] = min((lane + (uint32_t)k * L) * VEC, cols - VEC);
    rx[k] = VecIo<T, VEC>::template load<STREAM>(x + base + col[k]);
  }
  float z[K][VEC];
  if (bias) {
    const FastDiv period = {period_d, period_m, period_s};
    const size_t at = (size_t)(r - fast_div(r, period) * period_d) * cols;
#pragma unroll
    for (int k = 0; k < K; ++k) rb[k] = VecIo<T, VEC>::template load<false>(bias + at + col[k]);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float b[VEC];
      VecIo<T, VEC>::widen(rx[k], z[k]);
      VecIo<T, VEC>::widen(rb[k], b);
#pragma unroll
      for (int e = 0; e < VEC; ++e) z[k][e] += b[e];
    }
  } else {
#pragma unroll
    for (int k = 0; k < K; ++k) VecIo<T, VEC>::widen(rx[k], z[k]);
  }
  float most = 0.0f;
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int e = 0; e < VEC; ++e) most = fmaxf(most, __builtin_fabsf(z[k][e]));
  if constexpr (BLOCK) most = block_allreduce<OpMax>(most, slot, (int)(blockDim.x >> 6));
  else most = group_allreduce<OpMax>(most, (int)L);
  const Divisor s(scale_of(most, inv_max, tiny));
  if (row >= rows) return;
  if (lane == 0) scale[row] = s.s;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    if ((lane + (uint32_t)k * L) * VEC < cols) {
      float d[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) d[e] = s.divide(z[k][e]);
      VecIo<e4m3_t, VEC>::store(q + base + col[k], d);
      if constexpr (ACT != ACT_NONE) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) d[e] = activate<ACT>(z[k][e]);
        VecIo<T, VEC>::store(y + base + col[k], d);
      }
    }
  }
}

// Rows that no workgroup can hold: read twice, once for the maximum and once for the quotients.
template <typename T, int VEC, int ACT>
__global__ void __launch_bounds__(1024) k_checkpoint_long(const T* x, const T* bias, T* y, e4m3_t* q, float* scale, uint32_t rows, uint32_t cols,
                                                          int32_t, float inv_max, float tiny, uint32_t period_d, uint32_t period_m,
                                                          uint32_t period_s) {
  __shared__ float slot[16];
  const uint32_t row = blockIdx.x;
  const size_t base = (size_t)row * cols;
  const FastDiv period = {period_d, period_m, period_s};
  const size_t at = bias ? (size_t)(row - fast_div(row, period) * period_d) * cols : 0;
  auto values = [&](uint32_t c, float (&z)[VEC]) {
    VecIo<T, VEC>::widen(VecIo<T, VEC>::template load<false>(x + base + c), z);
    if (bias) {
      float b[VEC];
      VecIo<T, VEC>::widen(VecIo<T, VEC>::template load<false>(bias + at + c), b);
#pragma unroll
      for (int e = 0; e < VEC; ++e) z[e] += b[e];
    }
  };
  float most = 0.0f;
#pragma unroll 4
  for (uint32_t c = threadIdx.x * VEC; c < cols; c += 1024u * VEC) {
    float z[VEC];
    values(min(c, cols - VEC), z);
#pragma unroll
    for (int e = 0; e < VEC; ++e) most = fmaxf(most, __builtin_fabsf(z[e]));
  }
  const Divisor s(scale_of(block_allreduce<OpMax>(most, slot, 16), inv_max, tiny));
  if (threadIdx.x == 0) scale[row] = s.s;
#pragma unroll 2
  for (uint32_t c = threadIdx.x * VEC; c < cols; c += 1024u * VEC) {
    float z[VEC], d[VEC];
    const uint32_t col = min(c, cols - VEC);
    values(col, z);
#pragma unroll
    for (int e = 0; e < VEC; ++e) d[e] = s.divide(z[e]);
    VecIo<e4m3_t, VEC>::store(q + base + col, d);
    if constexpr (ACT != ACT_NONE) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) d[e] = activate<ACT>(z[e]);
      VecIo<T, VEC>::store(y + base + col, d);
    }
  }
}

// ---- use, element by element -------------------------------------------------------------------------------------------
// The tensor as one run of n values, block i of them at [i cols, (i + 1) cols).  With STRADDLE a lane's vector may reach into
// the next block (cols >= VEC, so it reaches into one at most, and n >= VEC).
template <typename T, int VEC, int ACT, bool STRADDLE, bool STREAM>
__global__ void __launch_bounds__(256) k_checkpoint_grad(const e4m3_t* q, const float* scale, const T* dy, T* out, uint32_t n, uint32_t cols_d,
                                                         uint32_t cols_m, uint32_t cols_s) {
  constexpr int U = 2;
  const FastDiv cols = {cols_d, cols_m, cols_s};
  const uint32_t first = (blockIdx.x * (256u * U) + threadIdx.x) * VEC;
  typename VecIo<e4m3_t, VEC>::Raw rq[U];
  typename VecIo<T, VEC>::Raw rd[U];
  float s0[U], s1[U];
  uint32_t at[U], edge[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    at[u] = min(first + (uint32_t)u * 256u * VEC, n - VEC);
    rq[u] = VecIo<e4m3_t, VEC>::template load<STREAM>(q + at[u]);
    if constexpr (ACT != ACT_NONE) rd[u] = VecIo<T, VEC>::template load<STREAM>(dy + at[u]);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t b = fast_div(at[u], cols);
    s0[u] = scale[b];
    if constexpr (STRADDLE) {
      edge[u] = (b + 1u) * cols_d - at[u];   // elements of the vector in block b (>= VEC: all)
      s1[u] = edge[u] < VEC ? scale[b + 1u] : 0.0f;
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float z[VEC], d[VEC];
    VecIo<e4m3_t, VEC>::widen(rq[u], z);
    if constexpr (ACT != ACT_NONE) VecIo<T, VEC>::widen(rd[u], d);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      z[e] *= STRADDLE && (uint32_t)e >= edge[u] ? s1[u] : s0[u];
      if constexpr (ACT != ACT_NONE) z[e] = d[e] * activation_slope<ACT>(z[e]);
    }
    if (first + (uint32_t)u * 256u * VEC < n) VecIo<T, VEC>::store(out + at[u], z);
  }
}

// ---- use, with column sums ---------------------------------------------------------------------------------------------
// Workgroup (ct, rb): 64 * VEC columns, row tiles rb, rb + n_rb, ... of WAVES * U rows.  A lane keeps its columns' sums in
// registers; the waves' are added in LDS in their order and go to the workspace, which K_COLFOLD folds.  `blocks` blocks of
// block_cols columns make up a row.  The loads of the next tile are under way while one is computed.
template <typename T, int VEC, int ACT, int WAVES, int U, bool STRADDLE, bool STREAM>
__global__ void __launch_bounds__(WAVES * 64) k_checkpoint_grad_sums(const e4m3_t* q, const float* scale, const T* dy, T* out, float* partials,
                                                                     uint32_t rows, uint32_t cols, uint32_t n_rb, uint32_t blocks,
                                                                     uint32_t block_cols, uint32_t pitch) {
  constexpr uint32_t TILE_COLS = 64 * VEC, TILE_ROWS = WAVES * U;
  __shared__ __align__(16) float red[WAVES][TILE_COLS];
  const uint32_t n_ct = (cols + TILE_COLS - 1) / TILE_COLS;
  const uint32_t rb = blockIdx.x / n_ct, ct = blockIdx.x - rb * n_ct;
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
  const uint32_t own = ct * TILE_COLS + lane * VEC;
  const uint32_t col = min(own, cols - VEC);   // (a lane past the end redoes the last columns and writes them again)
  const uint32_t b0 = col / block_cols;
  const uint32_t edge = (b0 + 1u) * block_cols - col;
  const uint32_t b1 = STRADDLE && edge < VEC ? b0 + 1u : b0;
  float acc[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) acc[e] = 0.0f;
  struct Row {
    typename VecIo<e4m3_t, VEC>::Raw q;
    typename VecIo<T, VEC>::Raw d;
    float s0, s1;
  };
  Row next[U], now[U];
  auto issue = [&](uint32_t r0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t r = min(r0 + wave + u * WAVES, rows - 1u);
      const size_t at = (size_t)r * cols + col;
      next[u].q = VecIo<e4m3_t, VEC>::template load<STREAM>(q + at);
      next[u].d = VecIo<T, VEC>::template load<STREAM>(dy + at);
      const float* s = scale + (size_t)r * blocks;
      next[u].s0 = s[b0];
      if constexpr (STRADDLE) next[u].s1 = s[b1];
    }
  };
  auto gradient = [&](const Row& w, float (&g)[VEC]) {
    float z[VEC];
    VecIo<e4m3_t, VEC>::widen(w.q, z);
    VecIo<T, VEC>::widen(w.d, g);
#pragma unroll
    for (int e = 0; e < VEC; ++e) g[e] *= activation_slope<ACT>(z[e] * (STRADDLE && (uint32_t)e >= edge ? w.s1 : w.s0));
  };
  const uint32_t stride = n_rb * TILE_ROWS;
  uint32_t r0 = rb * TILE_ROWS;
  issue(r0);   // (every workgroup has a row tile)
  for (; r0 < rows; r0 += stride) {
#pragma unroll
    for (int u = 0; u < U; ++u) now[u] = next[u];
    issue(r0 + stride);
    if (r0 + TILE_ROWS <= rows) {
      float g[U][VEC];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        gradient(now[u], g[u]);
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[e] += g[u][e];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) VecIo<T, VEC>::store(out + (size_t)(r0 + wave + u * WAVES) * cols + col, g[u]);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t r = r0 + wave + u * WAVES;
        if (r < rows) {
          float g[VEC];
          gradient(now[u], g);
#pragma unroll
          for (int e = 0; e < VEC; ++e) acc[e] += g[e];
          VecIo<T, VEC>::store(out + (size_t)r * cols + col, g);
        }
      }
    }
  }
  if constexpr (VEC == 1) {
    red[wave][lane] = acc[0];
  } else {
#pragma unroll
    for (int e = 0; e < VEC; e += 4) *reinterpret_cast<f32x4*>(&red[wave][lane * VEC + e]) = f32x4{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
  }
  __syncthreads();
  // column c of the tile: lane c / VEC had it, unless that lane's vector started early
  for (uint32_t c = threadIdx.x; c < TILE_COLS; c += WAVES * 64) {
    const uint32_t gc = ct * TILE_COLS + c;
    if (gc >= cols) break;
    const uint32_t first = min(gc - c % VEC, cols - VEC);
    const uint32_t slot = c / VEC * VEC + (gc - first);
    float s = red[0][slot];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) s += red[w][slot];
    partials[(size_t)rb * pitch + gc] = s;
  }
}

}  // namespace fsk

namespace fs {
using namespace fsk;

namespace {
template <typename T, int VEC, int ACT, bool S>
const void* store_sym(int32_t kernel, int vecs) {
  if (kernel == K_CHECKPOINT_LONG) return (const void*)k_checkpoint_long<T, VEC, ACT>;
  if constexpr (VEC == 1) return kernel == K_CHECKPOINT_WAVE && vecs == 1 ? (const void*)k_checkpoint<T, 1, 1, ACT, false, S> : nullptr;
  else if (kernel == K_CHECKPOINT_WAVE) {
    switch (vecs) {
      case 1: return (const void*)k_checkpoint<T, VEC, 1, ACT, false, S>;
      case 2: return (const void*)k_checkpoint<T, VEC, 2, ACT, false, S>;
      case 4: return (const void*)k_checkpoint<T, VEC, 4, ACT, false, S>;
      case 8: return (const void*)k_checkpoint<T, VEC, 8, ACT, false, S>;
    }
  } else {
    switch (vecs) {
      case 1: return (const void*)k_checkpoint<T, VEC, 1, ACT, true, S>;
      case 2: return (const void*)k_checkpoint<T, VEC, 2, ACT, true, S>;
      case 4: return (const void*)k_checkpoint<T, VEC, 4, ACT, true, S>;
    }
  }
  return nullptr;
}
template <typename T, int VEC, int ACT, bool STRADDLE, bool S>
const void* sums_sym(const CheckpointP& p) {
  if constexpr (ACT == ACT_NONE) return nullptr;
  else if (p.waves == 4 && p.unroll == 2) return (const void*)k_checkpoint_grad_sums<T, VEC, ACT, 4, 2, STRADDLE, S>;
  else if (p.waves == 4 && p.unroll == 4) return (const void*)k_checkpoint_grad_sums<T, VEC, ACT, 4, 4, STRADDLE, S>;
  else if (p.waves == 8 && p.unroll == 2) return (const void*)k_checkpoint_grad_sums<T, VEC, ACT, 8, 2, STRADDLE, S>;
  return nullptr;
}
template <typename T, int VEC, int ACT, bool S>
const void* act_sym(int32_t kernel, const CheckpointP& p) {
  const bool straddle = VEC > 1 && p.cols % VEC != 0;
  if (kernel == K_CHECKPOINT_GRAD)
    return straddle ? (const void*)k_checkpoint_grad<T, VEC, ACT, (VEC > 1), S> : (const void*)k_checkpoint_grad<T, VEC, ACT, false, S>;
  if (kernel == K_CHECKPOINT_GRAD_SUMS)
    return straddle && p.blocks > 1 ? sums_sym<T, VEC, ACT, (VEC > 1), S>(p) : sums_sym<T, VEC, ACT, false, S>(p);
  return store_sym<T, VEC, ACT, S>(kernel, p.vecs_per_lane);
}
template <typename T, int VEC, bool S>
const void* vec_sym(int32_t kernel, const CheckpointP& p) {
  switch (p.act) {
    case ACT_NONE: return act_sym<T, VEC, ACT_NONE, S>(kernel, p);
    case ACT_GELU: return act_sym<T, VEC, ACT_GELU, S>(kernel, p);
    case ACT_SILU: return act_sym<T, VEC, ACT_SILU, S>(kernel, p);
    default: return nullptr;
  }
}
template <typename T>
const void* type_sym(int32_t kernel, const CheckpointP& p) {
  if (p.vec == 1) return vec_sym<T, 1, false>(kernel, p);
  return p.stream ? vec_sym<T, Elem<T>::VEC, true>(kernel, p) : vec_sym<T, Elem<T>::VEC, false>(kernel, p);
}
}  // namespace

const void* checkpoint_kernel_symbol(int32_t kernel, const KernelArgs& a) {
  const CheckpointP& p = a.u.checkpoint;
  switch (p.dt) {
    case DT_F32: return type_sym<float>(kernel, p);
    case DT_F16: return type_sym<f16_t>(kernel, p);
    case DT_BF16: return type_sym<bf16_t>(kernel, p);
    default: return nullptr;
  }
}

}  // namespace fs
