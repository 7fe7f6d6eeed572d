// Pattern family: root-mean-square normalisation behind a residual connection (with a bias and a dropout in the branch that joins it),
// its result in 8 bits with a scale per row.
#include "fs_stitch_util.hpp"

namespace fs {

bool build_rmsnorm_8bit(const fs_graph& g, std::vector<Candidate>* out, PackForm*) {
  if (g.outputs.size() < 2 || g.outputs.size() > 5) return false;
  MatchState st;
  int32_t t_q = -1, t_s = -1;
  if (!match_8bit(g, "rmax[-1](abs($V))", &st, &t_q, &t_s)) return false;
  const int32_t tn = st.tensors["V"];
  if (!Pattern("mul(mul($H,rsqrt(addc[#0](rmean[-1](square($H))))),$G)").match(g, tn, &st)) return false;
  const int32_t th = st.tensors["H"], tg = st.tensors["G"];
  if (!is_input(g, tg)) return false;
  // the reciprocal deviation: the factor of h that is not h itself
  int32_t tr = -1;
  for (int k = 0; k < 2; ++k) {
    const int32_t t = g.ops[g.tensors[tn].producer].in[k];
    if (t == tg || is_input(g, t) || g.ops[g.tensors[t].producer].opcode != FS_MUL) continue;
    for (int j = 0; j < 2; ++j)
      if (g.ops[g.tensors[t].producer].in[j] != th) tr = g.ops[g.tensors[t].producer].in[j];
  }
  if (tr < 0) return false;

  // where h comes from
  RmsNorm8P p{};
  int32_t tsum = th, tx = th, tres = -1, tb = -1, t_state = -1, drop = -1;
  if (!is_input(g, th) && g.ops[g.tensors[th].producer].opcode == FS_CONVERT) {
    const Op& cv = g.ops[g.tensors[th].producer];
    st.covered.insert(g.tensors[th].producer);
    p.round_h = 1;
    p.dt = cv.to_dtype;   // has to be x's, checked below
    tsum = cv.in[0];
    tx = tsum;
    if (is_input(g, tsum)) return false;
  }
  if (!is_input(g, tsum)) {
    const int32_t add = g.tensors[tsum].producer;
    if (g.ops[add].opcode != FS_ADD) return false;
    st.covered.insert(add);
    // one operand is the residual, the other the branch: x, x + bias, or a dropout of one of them.  Both may be inputs.
    int32_t branch = -1;
    for (int k = 0; k < 2 && branch < 0; ++k) {
      const int32_t a = g.ops[add].in[k], b = g.ops[add].in[1 - k];
      if (!is_input(g, b) || !same_dims(g.tensors[b], g.tensors[tsum])) continue;
      if (!is_input(g, a) || same_dims(g.tensors[a], g.tensors[tsum])) {
        branch = a;
        tres = b;
      }
    }
    if (branch < 0) return false;
    p.form = 1;
    if (!is_input(g, branch) && Pattern("dropout($A,$STATE)").match(g, branch, &st)) {
      p.form = 2;
      drop = g.tensors[branch].producer;
      t_state = st.tensors["STATE"];
      branch = st.tensors["A"];
    }
    tx = branch;
    if (!is_input(g, branch)) {
      if (!Pattern("add($X,$B)").match(g, branch, &st)) return false;
      tx = st.tensors["X"];
      tb = st.tensors["B"];
      if (!is_input(g, tx) || !is_input(g, tb)) return false;
      if (!same_dims(g.tensors[tx], g.tensors[tsum])) std::swap(tx, tb);
    }
  }
  if (!covers_all(g, st)) return false;
  int32_t out_h = -1, out_n = -1, out_r = -1;
  for (int32_t t : g.outputs) {
    if (t == t_q || t == t_s) continue;
    if (t == th || (t == tsum && !p.round_h)) out_h = t;
    else if (t == tn) out_n = t;
    else if (t == tr) out_r = t;
    else return false;
  }

  // from here on the graph has the family's shape
  const Tensor& x = g.tensors[tx];
  const Tensor& gain = g.tensors[tg];
  if (p.round_h && p.dt != x.dtype) return true;
  p.dt = x.dtype;
  p.cols = (uint32_t)x.dims[x.rank - 1];
  p.rows = (uint32_t)(x.numel() / p.cols);
  p.wide_gamma = gain.dtype != p.dt ? 1 : 0;
  p.eps = (float)st.scalars[0];
  p.inv_cols = (float)(1.0 / (double)p.cols);
  p.inv_max = (float)st.scalars[80];
  p.tiny = (float)st.scalars[81];
  if (drop >= 0) p.draw = g.ops[drop].draw;
  p.stream = streams_inputs(g) ? 1 : 0;
  if (!is_float_dtype(p.dt) || !same_dims(x, g.tensors[th]) || !same_dims(x, g.tensors[tn])) return true;
  if (drop >= 0 && !same_dims(x, g.tensors[g.ops[drop].out])) return true;
  if (tres >= 0 && g.tensors[tres].dtype != p.dt) return true;
  if (tb >= 0 && (!is_row_vector(g.tensors[tb], p.cols) || g.tensors[tb].dtype != p.dt)) return true;
  if (!is_row_vector(gain, p.cols) || (gain.dtype != p.dt && gain.dtype != FS_F32)) return true;
  if (out_h >= 0 && g.tensors[out_h].store_as != p.dt) return true;
  if (out_n >= 0 && g.tensors[out_n].store_as != p.dt) return true;
  if (out_r >= 0 && g.tensors[out_r].store_as != FS_F32) return true;

  p.vec = p.cols >= (uint32_t)vec_of(p.dt) ? vec_of(p.dt) : 1;
  const int esz = dtype_bytes(p.dt);
  const double n = (double)p.rows * p.cols;
  const uint32_t nvec = (p.cols + p.vec - 1) / p.vec;
  const int wide = (tres >= 0 ? 2 : 1) + (out_h >= 0 ? 1 : 0) + (out_n >= 0 ? 1 : 0);
  auto start = [&](int32_t scheme, int32_t kernel) {
    Candidate c = make_candidate(g, "rmsnorm_8bit", scheme, kernel);
    Launch& l = c.launches.front();
    l.args.u.rms8 = p;
    l.ptr[0] = in_ref(g, tx);
    if (tres >= 0) l.ptr[1] = in_ref(g, tres);
    if (tb >= 0) l.ptr[2] = in_ref(g, tb);
    l.ptr[3] = in_ref(g, tg);
    if (t_state >= 0) l.ptr[4] = in_ref(g, t_state);
    if (out_h >= 0) l.ptr[5] = out_ref(g.tensors[out_h].output_slot);
    if (out_n >= 0) l.ptr[6] = out_ref(g.tensors[out_n].output_slot);
    l.ptr[7] = out_ref(g.tensors[t_q].output_slot);
    l.ptr[8] = out_ref(g.tensors[t_s].output_slot);
    if (out_r >= 0) l.ptr[9] = out_ref(g.tensors[out_r].output_slot);
    return c;
  };
  // The estimate (us), fitted to every candidate of 18,000 drawn shapes of 1 to 2^25 elements, three dtypes and all forms: on 9,000 others the
  // one chosen is 2.0 % behind the fastest (geometric mean; 1.4 % from 50 MB on).  Many values a lane leave too few wavefronts to keep the
  // memory busy (bf16 [8192,4096], 64 a lane 47.2, 32 43.4, 16 39.7, 8 39.6).  A workgroup's exchange shows with every round of resident
  // workgroups, and rows that are no whole vectors take a fifth more instructions and straddle lines.
  auto estimate = [&](KernelCost* kc, double lanes, int K, bool workgroup) {
    const double bytes = n * esz * wide + n + 4.0 * p.rows * (out_r >= 0 ? 2 : 1), whole = p.cols % p.vec == 0 ? 1.0 : 0.0;
    const double ops = (14.0 + (p.form == 2 ? 18.0 : 0.0) + (tb >= 0 ? 2.0 : 0.0)) * K * p.vec * (1.0 + 0.21 * (1.0 - whole));
    kc->vgpr_estimate = 24 + K * p.vec * (tres >= 0 ? 2 : 1) + K * p.vec;
    const double issue = std::max(1.0, kc->waves / 1024.0) * (31.1 + 3.54 * ops) / 2400.0;
    const double run = std::min<double>(lanes * p.vec, p.cols) * esz;
    const double per_simd = std::max(1, std::min(8, 512 / ((kc->vgpr_estimate + 7) / 8 * 8)));   // wavefronts
    const double memory = bytes / 7.75e6 * (1.0 + 0.017 * (1.0 / kc->lane_utilisation - 1.0)) * (1.0 + 0.367 * (8.0 / per_simd - 1.0)) *
                          (1.0 + 0.42 * std::max(0.0, 128.0 / run - whole));
    const double rounds = std::max(1.0, kc->waves / (1024.0 * per_simd)), exchange = workgroup ? rounds * (0.291 + 0.0287 * kc->waves_per_block) : 0.0;
    kc->own_estimate_s = (3.14 + std::pow(std::pow(memory, 1.49) + std::pow(issue, 1.49) + std::pow(exchange, 1.49), 1.0 / 1.49)) * 1e-6;
  };
  const char* form = p.form == 0 ? "plain" : p.form == 1 ? "residual" : "dropout";
  for (int K : {1, 2, 4, 8}) {
    const uint32_t L = pow2_at_least((nvec + K - 1) / K);
    if (L > 64 || (p.vec == 1 && K > 1)) continue;
    if (K > 1 && (uint64_t)L * K >= 2ull * nvec) continue;
    Candidate c = start(L == 1 ? FS_SCHEME_LOCAL : FS_SCHEME_WAVE, K_RMS8_WAVE);
    Launch& l = c.launches.front();
    l.args.u.rms8.lanes_log2 = log2_of(L);
    l.args.u.rms8.vecs_per_lane = K;
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
    snprintf(var, sizeof var, "<%s,%s,K%d,L%u>", dtype_name(p.dt), form, K, L);
    finish_candidate(&c, var, kc);
    out->push_back(c);
  }
  if (p.vec == 1) return true;
  for (int K : {1, 2, 4}) {
    const uint32_t T = std::max<uint32_t>(128, ((nvec + K - 1) / K + 63) / 64 * 64);
    if (T > 1024) continue;
    if ((uint64_t)T * K >= 2ull * nvec) continue;
    Candidate c = start(FS_SCHEME_LDS, K_RMS8_BLOCK);
    Launch& l = c.launches.front();
    l.args.u.rms8.vecs_per_lane = K;
    l.shape.block[0] = T;
    l.shape.grid[0] = p.rows;
    c.info.lanes_per_row = (int32_t)T;
    c.info.vecs_per_lane = K;
    c.info.rows_per_block = 1;
    c.info.lds_bytes = 256;
    KernelCost kc;
    kc.waves_per_block = (int32_t)(T / 64);
    kc.waves = (double)p.rows * kc.waves_per_block;
    kc.lds_bytes_per_block = 256;
    kc.lane_utilisation = (double)nvec / ((double)T * K);
    estimate(&kc, T, K, true);
    char var[48];
    snprintf(var, sizeof var, "<%s,%s,K%d,T%u>", dtype_name(p.dt), form, K, T);
    finish_candidate(&c, var, kc);
    out->push_back(c);
  }
  if (nvec > 4096) {   // what no workgroup holds
    Candidate c = start(FS_SCHEME_LDS, K_RMS8_LONG);
    Launch& l = c.launches.front();
    l.args.u.rms8.stream = 0;
    l.shape.block[0] = 1024;
    l.shape.grid[0] = p.rows;
    c.info.lanes_per_row = 1024;
    c.info.vecs_per_lane = 0;
    c.info.rows_per_block = 1;
    c.info.lds_bytes = 256;
    c.info.bytes_moved_model += (int64_t)(n * esz * (tres >= 0 ? 2 : 1));
    KernelCost kc;
    kc.waves_per_block = 16;
    kc.waves = (double)p.rows * 16;
    kc.lds_bytes_per_block = 256;
    estimate(&kc, 1024.0, 4, true);
    kc.own_estimate_s += 0.5 * n * esz * (tres >= 0 ? 2 : 1) / 6.3e12;   // the second reading finds a part of the row in the caches
    kc.own_estimate_s = std::max(kc.own_estimate_s, (2.0 + 2e-4 * p.cols) * 1e-6);
    char var[48];
    snprintf(var, sizeof var, "<%s,%s>", dtype_name(p.dt), form);
    finish_candidate(&c, var, kc);
    out->push_back(c);
  }
  return true;
}

}  // namespace fs
