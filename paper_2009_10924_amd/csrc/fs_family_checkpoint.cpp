// Pattern families: 8-bit activation checkpoints (alone, or with the bias and the activation that make them) and what the
// backward pass makes of them.
#include "fs_stitch_util.hpp"

namespace fs {

namespace {
// z = $Z -> an activation of it
const struct { const char* text; int32_t act; } kActivations[] = {{"gelu($Z)", ACT_GELU}, {"mul($Z,sigmoid($Z))", ACT_SILU}};
}  // namespace

bool match_activation(const fs_graph& g, int32_t t, MatchState* st, int32_t* act) {
  for (const auto& a : kActivations)
    if (Pattern(a.text).match(g, t, st)) {
      *act = a.act;
      return true;
    }
  return false;
}

// $Z's slope times $DY; SiLU's is s (1 + z (1 - s)) with s = sigmoid(z)
bool match_activation_gradient(const fs_graph& g, int32_t t, MatchState* st, int32_t* act) {
  MatchState trial = *st;
  if (Pattern("mul($DY,gelugrad($Z))").match(g, t, &trial)) {
    *act = ACT_GELU;
    *st = trial;
    return true;
  }
  trial = *st;
  if (Pattern("mul($DY,mul(sigmoid($Z),addc[#91](mul($Z,addc[#92](scale[#93](sigmoid($Z)))))))").match(g, t, &trial) && trial.scalars[91] == 1.0 &&
      trial.scalars[92] == 1.0 && trial.scalars[93] == -1.0) {
    *act = ACT_SILU;
    *st = trial;
    return true;
  }
  return false;
}

// The output that is $V's quotient by its scale, in 8 bits, and the scale: maxima of |$V| (`maximum` over "abs($V)"), times a
// constant, plus a constant.  Constants for which quotients by a reciprocal are those of a division (scales between 1e-37 and
// 2^125, whose reciprocals are normal numbers) and stay within the format's range (at least 1 / 448 of the maximum).
bool match_8bit(const fs_graph& g, const char* maximum, MatchState* st, int32_t* t_q, int32_t* t_s) {
  for (int32_t t : g.outputs) {
    if (g.tensors[t].store_as != FS_E4M3) continue;
    MatchState trial = *st;
    if (!Pattern(g.tensors[t].dtype == FS_E4M3 ? "cvt(div($V,$S))" : "div($V,$S)").match(g, t, &trial)) return false;
    const int32_t s = trial.tensors["S"];
    if (!Pattern("addc[#81](scale[#80](" + std::string(maximum) + "))").match(g, s, &trial)) return false;
    if (g.tensors[s].output_slot < 0 || g.tensors[s].store_as != FS_F32) return false;
    const double inv_max = trial.scalars[80], tiny = trial.scalars[81];
    if (!(inv_max >= (1.0 - 1e-6) / 448.0 && inv_max <= 0.125 && tiny >= 1e-37 && tiny <= 1e30)) return false;
    *st = trial;
    *t_q = t;
    *t_s = s;
    return true;
  }
  return false;
}

// A tensor that repeats along the leading axes of one of shape `full`: its extents are the trailing ones, those before them
// 1 or absent.
bool is_trailing(const Tensor& v, const Tensor& full) {
  if (v.rank > full.rank) return false;
  int k = 0;
  for (; k < v.rank && v.dims[v.rank - 1 - k] == full.dims[full.rank - 1 - k]; ++k) {}
  for (; k < v.rank; ++k)
    if (v.dims[v.rank - 1 - k] != 1) return false;
  return true;
}

namespace {
// blocks of `cols` values: how many values a lane accesses at once
int access_of(int32_t dt, uint32_t cols) { return cols >= (uint32_t)vec_of(dt) ? vec_of(dt) : 1; }
}  // namespace

// ------------------------------------------------------------------ store
bool build_checkpoint(const fs_graph& g, std::vector<Candidate>* out, PackForm*) {
  if (g.outputs.size() != 2 && g.outputs.size() != 3) return false;
  MatchState st;
  int32_t t_q = -1, t_s = -1, t_y = -1, act = ACT_NONE;
  if (!match_8bit(g, "rmax[-1](abs($V))", &st, &t_q, &t_s)) return false;
  const int32_t tz = st.tensors["V"];
  st.tensors["Z"] = tz;
  for (int32_t t : g.outputs) {
    if (t == t_q || t == t_s) continue;
    if (t_y >= 0 || !match_activation(g, t, &st, &act)) return false;
    t_y = t;
  }
  int32_t tx = tz, tb = -1;
  if (!is_input(g, tz)) {
    if (!Pattern("add($X,$B)").match(g, tz, &st)) return false;
    tx = st.tensors["X"];
    tb = st.tensors["B"];
    if (!is_input(g, tx) || !is_input(g, tb)) return false;
    if (!same_dims(g.tensors[tx], g.tensors[tz])) std::swap(tx, tb);
  }
  if (!covers_all(g, st)) return false;
  const Tensor& x = g.tensors[tx];
  CheckpointP p{};
  p.dt = x.dtype;
  p.act = act;
  p.cols = (uint32_t)x.dims[x.rank - 1];
  p.rows = (uint32_t)(x.numel() / p.cols);
  p.blocks = 1;
  p.inv_max = (float)st.scalars[80];
  p.tiny = (float)st.scalars[81];
  p.stream = streams_inputs(g) ? 1 : 0;
  p.vec = access_of(p.dt, p.cols);
  if (!is_float_dtype(p.dt) || !same_dims(x, g.tensors[tz])) return true;
  if (t_y >= 0 && g.tensors[t_y].store_as != p.dt) return true;
  uint32_t period = 1;
  if (tb >= 0) {
    const Tensor& b = g.tensors[tb];
    if (b.dtype != p.dt || !is_trailing(b, x) || b.dims[b.rank - 1] != (int64_t)p.cols) return true;
    period = (uint32_t)(b.numel() / p.cols);
  }
  p.div_period = make_fastdiv(period);
  if (p.div_period.d == 0) return true;

  const int esz = dtype_bytes(p.dt);
  const double n = (double)p.rows * p.cols;
  const uint32_t nvec = (p.cols + p.vec - 1) / p.vec;
  auto fill_ptrs = [&](Launch& l) {
    l.ptr[0] = in_ref(g, tx);
    if (tb >= 0) l.ptr[1] = in_ref(g, tb);
    if (t_y >= 0) l.ptr[2] = out_ref(g.tensors[t_y].output_slot);
    l.ptr[3] = out_ref(g.tensors[t_q].output_slot);
    l.ptr[4] = out_ref(g.tensors[t_s].output_slot);
  };
  // The estimate of a launch (us), fitted to every candidate of 360 shapes of 1 to 2^26 values, three dtypes: the one chosen is 1.0 %
  // behind the fastest on 50 others (geometric mean; 2.7 % by the general evaluator, which knows nothing of 8-bit stores, whose runs are the
  // shortest of a lane group's).  A step of few lanes writes a part of a line; rows that are no multiple of an access end inside one.
  auto estimate = [&](KernelCost* kc, double lanes, int K, bool workgroup) {
    const double bytes = n * esz * (t_y >= 0 ? 2 : 1) + n + 4.0 * p.rows;
    const double ops = (5.0 + 5.0 * (act == ACT_GELU ? 1.5 : act == ACT_SILU ? 1.0 : 0.0) + (tb >= 0 ? 1.0 : 0.0)) * K * p.vec;
    const double issue = std::max(1.0, kc->waves / 1024.0) * (0.183 + 1.14e-3 * ops);
    const double run = std::min<double>(lanes * p.vec, p.cols);
    double memory = bytes / 6.4e6 * (1.0 + 0.171 * (1.0 / kc->lane_utilisation - 1.0));
    if (p.cols % p.vec == 0 && p.cols % 16 == 0) memory *= 1.0 + 0.115 * std::max(0.0, 128.0 / run - 1.0);
    else memory *= 1.0 + 0.012 * std::max(0.0, 512.0 / run - 1.0) + (K * p.vec > 8 ? 0.043 : 0.0);
    if (K * p.vec >= 64) memory *= 1.18;   // more than 128 registers
    kc->own_estimate_s = (3.1 + (workgroup ? 0.41 : 0.0) + std::max(issue, memory)) * 1e-6;
    kc->vgpr_estimate = 24 + K * p.vec * 2;
  };
  for (int K : {1, 2, 4, 8}) {
    const uint32_t L = pow2_at_least((nvec + K - 1) / K);
    if (L > 64 || (p.vec == 1 && K > 1)) continue;
    if (K > 1 && (uint64_t)L * K >= 2ull * nvec) continue;
    Candidate c = make_candidate(g, "checkpoint", L == 1 ? FS_SCHEME_LOCAL : FS_SCHEME_WAVE, K_CHECKPOINT_WAVE);
    Launch& l = c.launches.front();
    CheckpointP& q = l.args.u.checkpoint;
    q = p;
    q.lanes_log2 = log2_of(L);
    q.vecs_per_lane = K;
    fill_ptrs(l);
    l.shape.block[0] = 256;
    l.shape.grid[0] = (p.rows + 256 / L - 1) / (256 / L);
    c.info.lanes_per_row = (int32_t)L;
    c.info.vecs_per_lane = K;
    c.info.rows_per_block = (int32_t)(256 / L);
    KernelCost kc;
    kc.waves = (double)l.shape.grid[0] * 4;
    kc.waves_per_block = 4;
    kc.lane_utilisation = (double)nvec / ((double)L * K);
    estimate(&kc, L, K, false);
    char var[48];
    snprintf(var, sizeof var, "<%s,%s,K%d,L%u>", dtype_name(p.dt), act_name(act), K, L);
    finish_candidate(&c, var, kc);
    out->push_back(c);
  }
  if (p.vec == 1) return true;
  for (int K : {1, 2, 4}) {
    const uint32_t T = std::max<uint32_t>(128, ((nvec + K - 1) / K + 63) / 64 * 64);
    if (T > 1024) continue;
    if ((uint64_t)T * K >= 2ull * nvec) continue;
    Candidate c = make_candidate(g, "checkpoint", FS_SCHEME_LDS, K_CHECKPOINT_BLOCK);
    Launch& l = c.launches.front();
    CheckpointP& q = l.args.u.checkpoint;
    q = p;
    q.vecs_per_lane = K;
    fill_ptrs(l);
    l.shape.block[0] = T;
    l.shape.grid[0] = p.rows;
    c.info.lanes_per_row = (int32_t)T;
    c.info.vecs_per_lane = K;
    c.info.rows_per_block = 1;
    c.info.lds_bytes = 64;
    KernelCost kc;
    kc.waves_per_block = (int32_t)(T / 64);
    kc.waves = (double)p.rows * kc.waves_per_block;
    kc.lds_bytes_per_block = 64;
    kc.lane_utilisation = (double)nvec / ((double)T * K);
    estimate(&kc, T, K, true);
    char var[48];
    snprintf(var, sizeof var, "<%s,%s,K%d,T%u>", dtype_name(p.dt), act_name(act), K, T);
    finish_candidate(&c, var, kc);
    out->push_back(c);
  }
  if (nvec > 4096) {   // what no workgroup holds
    Candidate c = make_candidate(g, "checkpoint", FS_SCHEME_LDS, K_CHECKPOINT_LONG);
    Launch& l = c.launches.front();
    l.args.u.checkpoint = p;
    l.args.u.checkpoint.stream = 0;
    fill_ptrs(l);
    l.shape.block[0] = 1024;
    l.shape.grid[0] = p.rows;
    c.info.lanes_per_row = 1024;
    c.info.vecs_per_lane = 0;
    c.info.rows_per_block = 1;
    c.info.lds_bytes = 64;
    c.info.bytes_moved_model += (int64_t)(n * esz);
    KernelCost kc;
    kc.waves_per_block = 16;
    kc.waves = (double)p.rows * 16;
    kc.lds_bytes_per_block = 64;
    estimate(&kc, 1024.0, 4, true);
    kc.own_estimate_s += 0.5 * n * esz / 6.4e12;   // the second read finds a part of the row in the caches
    // A compute unit by itself takes a block at 4500 to 10800 values a us, 2-byte and 4-byte ones alike (bf16 [1, 2^26] 7677 us, with bias and
    // GELU [1, 2^22] 950, f32 [1, 2^22] 511, with GELU [16, 2^18] 43): what fewer blocks than compute units take.
    const double per_value = 1.05e-4 + 0.45e-4 * (act == ACT_GELU ? 1.5 : act == ACT_SILU ? 1.0 : 0.0) + (tb >= 0 ? 0.5e-4 : 0.0);
    kc.own_estimate_s = std::max(kc.own_estimate_s, (2.0 + per_value * p.cols) * 1e-6);
    char var[48];
    snprintf(var, sizeof var, "<%s,%s>", dtype_name(p.dt), act_name(act));
    finish_candidate(&c, var, kc);
    out->push_back(c);
  }
  return true;
}

// ------------------------------------------------------------------ use
bool build_checkpoint_backward(const fs_graph& g, std::vector<Candidate>* out, PackForm*) {
  if (!holds_8bit(g) || g.outputs.empty() || g.outputs.size() > 2) return false;
  MatchState st;
  int32_t act = ACT_NONE, t_out = -1, t_sum = -1;
  // the sum over all rows, if there is one: reduce_sums along each leading axis but those of the row, in turn
  for (int32_t t : g.outputs) {
    const Tensor& T = g.tensors[t];
    if (T.producer >= 0 && g.ops[T.producer].opcode == FS_REDUCE_SUM) {
      if (t_sum >= 0) return false;
      t_sum = t;
    } else {
      if (t_out >= 0) return false;
      t_out = t;
    }
  }
  if (t_out < 0) return false;
  int summed_axes = 0;
  if (t_sum >= 0) {
    int32_t t = t_sum;
    uint32_t axes = 0;
    while (t != t_out) {
      const Tensor& T = g.tensors[t];
      if (T.producer < 0 || g.ops[T.producer].opcode != FS_REDUCE_SUM || (t != t_sum && T.output_slot >= 0)) return false;
      axes |= 1u << g.ops[T.producer].axis;
      st.covered.insert(T.producer);
      t = g.ops[T.producer].in[0];
    }
    while ((axes >> summed_axes) & 1u) ++summed_axes;
    if (axes != (1u << summed_axes) - 1u) return false;   // not the leading ones
  }
  if (match_activation_gradient(g, t_out, &st, &act)) {
    if (!is_input(g, st.tensors["DY"])) return false;
  } else {
    if (t_sum >= 0) return false;
    st.tensors["Z"] = t_out;
  }
  if (!Pattern("mul($Q,$S)").match(g, st.tensors["Z"], &st) || !covers_all(g, st)) return false;
  int32_t tq = st.tensors["Q"], ts = st.tensors["S"];
  if (g.tensors[tq].dtype != FS_E4M3) std::swap(tq, ts);
  if (!is_input(g, tq) || !is_input(g, ts) || g.tensors[tq].dtype != FS_E4M3) return false;
  const Tensor& q = g.tensors[tq];
  const Tensor& s = g.tensors[ts];
  const int32_t tdy = act != ACT_NONE ? st.tensors["DY"] : -1;
  CheckpointP p{};
  p.dt = g.tensors[t_out].store_as;
  p.act = act;
  p.cols = (uint32_t)q.dims[q.rank - 1];
  p.rows = (uint32_t)(q.numel() / p.cols);
  p.blocks = 1;
  p.stream = streams_inputs(g) ? 1 : 0;
  p.vec = access_of(p.dt, p.cols);
  // one scale per block of the last axis: q's extents but for the last (others of as many values would stretch q with them)
  Tensor scales = q;
  scales.dims[q.rank - 1] = 1;
  if (!is_float_dtype(p.dt) || s.dtype != FS_F32 || !same_dims(s, scales)) return true;
  if (tdy >= 0 && (!same_dims(g.tensors[tdy], q) || g.tensors[tdy].dtype != p.dt)) return true;
  const int esz = dtype_bytes(p.dt);
  const double n = (double)p.rows * p.cols;
  KernelCost base;
  base.hbm_bytes = n + 4.0 * p.rows + n * esz * (tdy >= 0 ? 2 : 1);
  base.elems = n;
  base.valu_per_elem = 4.0 + (act == ACT_NONE ? 0.0 : 5.0 + act_valu(act)) + (p.cols % p.vec != 0 ? 2.0 : 0.0);
  base.trans_per_elem = act_trans(act);
  base.cache_bytes = n / p.vec * 4.0;

  if (t_sum < 0) {
    p.div_cols = make_fastdiv(p.cols);
    if (p.div_cols.d == 0) return true;
    Candidate c = make_candidate(g, "checkpoint_backward", FS_SCHEME_LOCAL, K_CHECKPOINT_GRAD);
    Launch& l = c.launches.front();
    l.args.u.checkpoint = p;
    l.ptr[0] = in_ref(g, tq);
    l.ptr[1] = in_ref(g, ts);
    if (tdy >= 0) l.ptr[2] = in_ref(g, tdy);
    l.ptr[3] = out_ref(g.tensors[t_out].output_slot);
    l.shape.block[0] = 256;
    l.shape.grid[0] = (uint32_t)((n + 512.0 * p.vec - 1) / (512.0 * p.vec));
    c.info.vecs_per_lane = 2;
    KernelCost kc = base;
    kc.waves = (double)l.shape.grid[0] * 4;
    kc.waves_per_block = 4;
    kc.bytes_in_flight_per_lane = 2.0 * p.vec * (1 + (tdy >= 0 ? esz : 0));
    kc.vgpr_estimate = 40;
    char var[48];
    snprintf(var, sizeof var, "<%s,%s>", dtype_name(p.dt), act_name(act));
    finish_candidate(&c, var, kc);
    out->push_back(c);
    return true;
  }

  if (g.tensors[t_sum].store_as != FS_F32) return true;
  for (int k = summed_axes; k < q.rank - 1; ++k) p.blocks *= (uint32_t)q.dims[k];
  p.rows /= p.blocks;
  if (summed_axes == q.rank) return true;   // summed along the row as well
  const uint32_t cols = p.blocks * p.cols;
  const uint32_t tile_cols = 64 * (uint32_t)p.vec;
  const uint32_t n_col_tiles = (cols + tile_cols - 1) / tile_cols;
  struct Shape { int waves, unroll; };
  for (Shape sh : {Shape{4, 2}, Shape{4, 4}, Shape{8, 2}}) {
    const uint32_t tile_rows = sh.waves * sh.unroll;
    const uint32_t max_rb = (p.rows + tile_rows - 1) / tile_rows;
    uint32_t last_rb = 0;
    for (uint32_t want : {0u, 128u, 256u}) {
      // enough workgroups to fill the chip, few enough that the partial sums stay small; or one on all of few rows of its columns,
      // whose sums are complete: a launch less, but a compute unit reads no faster for being alone (bf16 rows of 4096: 16 rows 6.9 ->
      // 3.7 us, 33 6.6 -> 4.6, 64 level, 128 6.6 -> 11.7)
      if (want == 0 && p.rows > 48) continue;
      const uint32_t n_rb = std::min(max_rb, std::max<uint32_t>(1, want * 6 / n_col_tiles));
      if (n_rb == last_rb) continue;
      last_rb = n_rb;
      const bool fold = n_rb > 1;
      Candidate c = make_candidate(g, "checkpoint_backward", FS_SCHEME_GLOBAL, K_CHECKPOINT_GRAD_SUMS);
      const uint32_t pitch = colsum_pitch(cols);
      {
        Launch& l = c.launches.front();
        CheckpointP& k = l.args.u.checkpoint;
        k = p;
        k.waves = sh.waves;
        k.unroll = sh.unroll;
        k.n_row_blocks = n_rb;
        l.ptr[0] = in_ref(g, tq);
        l.ptr[1] = in_ref(g, ts);
        l.ptr[2] = in_ref(g, tdy);
        l.ptr[3] = out_ref(g.tensors[t_out].output_slot);
        l.ptr[4] = fold ? ws_ref(0) : out_ref(g.tensors[t_sum].output_slot);
        l.shape.block[0] = sh.waves * 64;
        l.shape.grid[0] = n_rb * n_col_tiles;
      }
      if (fold) {
        c.launches.emplace_back();
        Launch& f = c.launches.back();
        make_fold_launch(&f, n_rb, pitch, pitch, cols);
        f.ptr[0] = ws_ref(0);
        f.ptr[1] = out_ref(g.tensors[t_sum].output_slot);
        c.info.n_kernels = 2;
        c.info.workspace_bytes = (int64_t)n_rb * pitch * 4;
      }
      c.info.rows_per_block = (int32_t)tile_rows;
      c.info.vecs_per_lane = sh.unroll;
      c.info.lanes_per_row = 64;
      c.info.lds_bytes = sh.waves * (int32_t)tile_cols * 4;
      c.info.bytes_moved_model = c.info.bytes_min + 2 * c.info.workspace_bytes;
      KernelCost kc = base;
      kc.partial_bytes = 2.0 * (double)c.info.workspace_bytes;
      kc.fold_rows = fold ? n_rb : 0;
      kc.flush_values = p.vec;
      kc.flush_steps = 0;
      kc.waves_per_block = sh.waves;
      kc.waves = (double)n_rb * n_col_tiles * sh.waves;
      kc.bytes_in_flight_per_lane = (double)p.vec * (1 + esz) * sh.unroll;
      kc.vgpr_estimate = 40 + 14 * sh.unroll;
      kc.barriers = 1;
      kc.lds_bytes_per_block = c.info.lds_bytes;
      kc.rows_per_wave_loop = std::max(1.0, (double)p.rows / ((double)n_rb * tile_rows));
      kc.access_run_bytes = 64.0 * p.vec * esz;
      kc.row_bytes = (double)cols * esz;
      kc.dep_phases = 0;
      char var[56];
      snprintf(var, sizeof var, "<%s,%s,W%d,U%d,RB%u%s>", dtype_name(p.dt), act_name(act), sh.waves, sh.unroll, n_rb, fold ? ",fold" : "");
      finish_candidate(&c, var, kc);
      out->push_back(c);
    }
  }
  return true;
}

}  // namespace fs
