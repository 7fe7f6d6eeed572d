// Pattern family: dropout with the bias and activation in front of it and the residual behind it, and its backward pass with the
// activation's slope.  (Behind or in front of row reductions, and with column sums, a dropout is part of a row program.)
#include "fs_stitch_util.hpp"

namespace fs {

namespace {
// $Z is an input, or one with a bias per column: its ops join st->covered
bool match_biased(const fs_graph& g, int32_t tz, MatchState* st, int32_t* tx, int32_t* tb) {
  *tx = tz;
  *tb = -1;
  if (is_input(g, tz)) return true;
  if (!Pattern("add($X,$B)").match(g, tz, st)) return false;
  *tx = st->tensors["X"];
  *tb = st->tensors["B"];
  if (!is_input(g, *tx) || !is_input(g, *tb)) return false;
  if (!same_dims(g.tensors[*tx], g.tensors[tz])) std::swap(*tx, *tb);
  return true;
}
}  // namespace

bool build_dropout(const fs_graph& g, std::vector<Candidate>* out, PackForm*) {
  if (g.outputs.size() != 1) return false;
  const int32_t ty = g.outputs[0];
  MatchState st;
  int32_t act = ACT_NONE, t_other = -1, tz = -1, t_state = -1, drop = -1;
  const bool slope = match_activation_gradient(g, ty, &st, &act);
  if (slope) {
    MatchState more = st;
    const int32_t t = st.tensors["DY"];
    if (!Pattern("dropout($D,$STATE)").match(g, t, &more)) return false;
    st = more;
    drop = g.tensors[t].producer;
    t_other = st.tensors["D"];
    tz = st.tensors["Z"];
  } else {
    int32_t t = ty;
    const int32_t add = g.tensors[ty].producer;
    if (g.ops[add].opcode == FS_ADD) {
      for (int k = 0; k < 2 && t == ty; ++k) {
        const int32_t a = g.ops[add].in[k], b = g.ops[add].in[1 - k];
        if (is_input(g, b) && !is_input(g, a) && g.ops[g.tensors[a].producer].opcode == FS_DROPOUT) {
          t = a;
          t_other = b;
        }
      }
      if (t == ty) return false;
      st.covered.insert(add);
    }
    if (!Pattern("dropout($A,$STATE)").match(g, t, &st)) return false;
    drop = g.tensors[t].producer;
    tz = st.tensors["A"];
    if (!is_input(g, tz) && match_activation(g, tz, &st, &act)) tz = st.tensors["Z"];
  }
  t_state = st.tensors["STATE"];
  int32_t tx = -1, tb = -1;
  if (!match_biased(g, tz, &st, &tx, &tb) || !covers_all(g, st)) return false;
  if (t_other >= 0 && !is_input(g, t_other)) return false;
  const Tensor& x = g.tensors[tx];
  DropoutP p{};
  p.in_dt = p.out_dt = x.dtype;
  p.act = act;
  p.slope = slope ? 1 : 0;
  p.has_other = t_other >= 0 ? 1 : 0;
  p.cols = (uint32_t)x.dims[x.rank - 1];
  p.rows = (uint32_t)(x.numel() / p.cols);
  p.div_groups = make_fastdiv((p.cols + 7) / 8);
  p.draw = g.ops[drop].draw;
  p.stream = streams_inputs(g) ? 1 : 0;
  // the dropout's own operand has the tensor's extents (a residual or gradient that stretches it is another pattern)
  if (!is_float_dtype(p.in_dt) || !same_dims(x, g.tensors[ty]) || g.tensors[ty].store_as != p.in_dt || !same_dims(x, g.tensors[g.ops[drop].out])) return true;
  if (t_other >= 0 && (!same_dims(g.tensors[t_other], x) || g.tensors[t_other].dtype != p.in_dt)) return true;
  if (tb >= 0 && (!is_row_vector(g.tensors[tb], p.cols) || g.tensors[tb].dtype != p.in_dt)) return true;
  if (p.div_groups.d == 0) return true;

  const int esz = dtype_bytes(p.in_dt);
  const double n = (double)p.rows * p.cols;
  Candidate c = make_candidate(g, "dropout", FS_SCHEME_LOCAL, K_DROPOUT);
  Launch& l = c.launches.front();
  l.args.u.dropout = p;
  l.ptr[0] = in_ref(g, tx);
  if (tb >= 0) l.ptr[1] = in_ref(g, tb);
  if (t_other >= 0) l.ptr[2] = in_ref(g, t_other);
  l.ptr[3] = in_ref(g, t_state);
  l.ptr[4] = out_ref(0);
  const uint64_t groups = (uint64_t)p.rows * p.div_groups.d;
  l.shape.block[0] = 256;
  l.shape.grid[0] = (uint32_t)((groups + 255) / 256);
  c.info.vecs_per_lane = 8 / vec_of(p.in_dt);
  KernelCost kc;
  kc.waves = (double)l.shape.grid[0] * 4;
  kc.waves_per_block = 4;
  kc.lane_utilisation = (double)p.cols / (8.0 * p.div_groups.d);
  kc.vgpr_estimate = 48;
  // memory, or the generator (13 operations for each of its eight numbers) and what is beside it
  const double ops = (20.0 + act_valu(act) + 4.0 * act_trans(act)) * (double)groups * 8.0;
  kc.own_estimate_s = 3.0e-6 + std::max(n * esz * (t_other >= 0 ? 3 : 2) / 6.3e12, ops / 3.4e13);
  char var[48];
  snprintf(var, sizeof var, "<%s,%s%s%s>", dtype_name(p.in_dt), act_name(act), slope ? ",slope" : "", p.cols % 8 != 0 ? ",ragged" : "");
  finish_candidate(&c, var, kc);
  out->push_back(c);
  return true;
}

}  // namespace fs
