// Pattern family: rotary positions of one tensor, or of two (queries and keys) at the same positions, with transposes of the leading
// axes in front of or behind them (head split and merge) folded into where rows are read and written.
#include "fs_stitch_util.hpp"

namespace fs {

namespace {
struct Rotated {
  int32_t op = -1, in = -1, out = -1;   // the rotary op; the graph input it reads; the graph output
  uint32_t in_stride[3], out_stride[3]; // elements, along the rotary operand's leading axes
};

// Row strides (elements) of `t`'s leading axes, its extents right-aligned to three.
void leading_strides(const Tensor& t, uint32_t (&s)[3]) {
  int64_t acc = t.dims[t.rank - 1];
  for (int k = 0; k < 3; ++k) s[k] = 0;
  for (int k = t.rank - 2; k >= 0; --k) {
    s[3 - (t.rank - 1) + k] = (uint32_t)acc;
    acc *= t.dims[k];
  }
}

// output `t`: a rotary op's result, or that rounded and transposed; the op's operand: a graph input, or one transposed
bool trace(const fs_graph& g, int32_t t, Rotated* r, size_t* covered) {
  r->out = t;
  const Op* back = nullptr;
  int32_t y = t;
  if (g.ops[g.tensors[t].producer].opcode == FS_TRANSPOSE) {
    back = &g.ops[g.tensors[t].producer];
    y = back->in[0];
    ++*covered;
    if (is_input(g, y) || g.tensors[y].output_slot >= 0 || g.tensors[y].consumers.size() != 1) return false;
    // (a transpose moves values as they are stored, so the rounding stands in front of it)
    if (g.ops[g.tensors[y].producer].opcode == FS_CONVERT && g.ops[g.tensors[y].producer].to_dtype == g.tensors[t].store_as) {
      y = g.ops[g.tensors[y].producer].in[0];
      ++*covered;
      if (is_input(g, y) || g.tensors[y].output_slot >= 0 || g.tensors[y].consumers.size() != 1) return false;
    }
  }
  if (g.ops[g.tensors[y].producer].opcode != FS_ROTARY) return false;
  r->op = g.tensors[y].producer;
  ++*covered;
  const Op& op = g.ops[r->op];
  if (!is_input(g, op.in[1])) return false;
  const Op* forth = nullptr;
  int32_t x = op.in[0];
  if (!is_input(g, x)) {
    if (g.ops[g.tensors[x].producer].opcode != FS_TRANSPOSE || g.tensors[x].output_slot >= 0 || g.tensors[x].consumers.size() != 1) return false;
    forth = &g.ops[g.tensors[x].producer];
    ++*covered;
    x = forth->in[0];
    if (!is_input(g, x)) return false;
  }
  r->in = x;
  const int rank = g.tensors[y].rank;
  for (const Op* tr : {back, forth})
    if (tr && tr->perm[rank - 1] != rank - 1) return false;   // elements of a row would part
  uint32_t s[3];
  leading_strides(g.tensors[x], s);
  for (int k = 0; k < 3; ++k) r->in_stride[k] = s[k];
  if (forth)
    for (int k = 0; k < rank - 1; ++k) r->in_stride[3 - (rank - 1) + k] = s[3 - (rank - 1) + forth->perm[k]];
  leading_strides(g.tensors[t], s);
  for (int k = 0; k < 3; ++k) r->out_stride[k] = s[k];
  if (back)
    for (int k = 0; k < rank - 1; ++k) r->out_stride[3 - (rank - 1) + back->perm[k]] = s[3 - (rank - 1) + k];
  return true;
}
}  // namespace

bool build_rotary(const fs_graph& g, std::vector<Candidate>* out, PackForm*) {
  if (g.outputs.empty() || g.outputs.size() > 2) return false;
  const size_t tensors = g.outputs.size();
  Rotated r[2];
  size_t covered = 0;
  for (size_t i = 0; i < tensors; ++i)
    if (!trace(g, g.outputs[i], &r[i], &covered)) return false;
  if (covered != g.ops.size()) return false;
  const Op& first = g.ops[r[0].op];
  const int32_t t_pos = first.in[1];
  if (tensors == 2) {
    const Op& second = g.ops[r[1].op];
    const fs_attr_rotary &a = first.rotary, &b = second.rotary;
    bool same = second.in[1] == t_pos && a.base == b.base && a.n_axes == b.n_axes && a.interleaved == b.interleaved && a.restart == b.restart &&
                a.inverse == b.inverse;
    for (int k = 0; same && k < a.n_axes; ++k) same = a.pairs[k] == b.pairs[k];
    const Tensor &x = g.tensors[first.in[0]], &y = g.tensors[second.in[0]];
    if (!same || x.rank != y.rank || x.dims[x.rank - 1] != y.dims[y.rank - 1] || x.dtype != y.dtype) return false;
  }
  const Tensor& x0 = g.tensors[first.in[0]];
  const Tensor& pos = g.tensors[t_pos];
  RotaryP p{};
  p.in_dt = p.out_dt = x0.dtype;
  p.interleaved = first.rotary.interleaved;
  p.stream = streams_inputs(g) ? 1 : 0;
  RotaryShape& s = p.s;
  s.angles = rotary_angles(first.rotary);
  s.dim = (uint32_t)x0.dims[x0.rank - 1];
  if (!is_float_dtype(p.in_dt)) return true;
  for (size_t i = 0; i < tensors; ++i)
    if (g.tensors[r[i].out].store_as != p.in_dt) return true;
  // axes along which the positions vary, and those that they stretch over
  uint32_t pos_ext[3] = {1, 1, 1}, step = 1;
  for (int k = 1; k < pos.rank; ++k) {
    const uint32_t d = (uint32_t)pos.dims[pos.rank - 1 - k];
    pos_ext[3 - k] = d;
    s.pos_stride[3 - k] = d == 1 ? 0 : step;
    step *= d;
  }
  s.positions = step;
  s.pos_div[0] = make_fastdiv(pos_ext[2]);
  s.pos_div[1] = make_fastdiv(pos_ext[1]);
  uint32_t shared = 0;
  for (size_t i = 0; i < 2; ++i) {
    RotaryRows& t = s.t[i];
    uint32_t ext[3] = {1, 1, 1};
    t.shared = 0;
    if (i < tensors) {
      const Tensor& x = g.tensors[g.ops[r[i].op].in[0]];
      t.shared = 1;
      for (int k = 0; k < x.rank - 1; ++k) {
        const int at = 3 - (x.rank - 1) + k;
        if (pos_ext[at] == 1) ext[at] = (uint32_t)x.dims[k];
        t.shared *= ext[at];
      }
      for (int k = 0; k < 3; ++k) t.in_stride[k] = r[i].in_stride[k], t.out_stride[k] = r[i].out_stride[k];
    }
    t.div[0] = make_fastdiv(ext[2]);
    t.div[1] = make_fastdiv(ext[1]);
    if (t.div[0].d == 0 || t.div[1].d == 0) return true;
    shared += t.shared;
  }
  // neighbouring rows of memory are at neighbouring positions where the innermost leading axis has its own
  s.p_inner = pos_ext[2] > 1 ? 1 : 0;
  const uint32_t rest = s.dim - 2 * s.angles.pairs;
  const uint32_t V = (uint32_t)vec_of(p.in_dt);
  const uint32_t turned = p.interleaved ? 2 * s.angles.pairs : s.angles.pairs;   // elements that the accesses of turning steps start in
  p.vec = turned >= V && (rest == 0 || rest >= V) ? (int32_t)V : 1;
  const uint32_t vec = (uint32_t)p.vec;
  s.rot_units = vec == 1 ? s.angles.pairs : (turned + vec - 1) / vec;
  const uint32_t units = s.rot_units + (rest + vec - 1) / vec;
  s.div_units = make_fastdiv(units);
  if (s.pos_div[0].d == 0 || s.pos_div[1].d == 0 || s.div_units.d == 0) return true;

  const int esz = dtype_bytes(p.in_dt);
  double n = 0;
  for (size_t i = 0; i < tensors; ++i) n += (double)g.tensors[r[i].out].numel();
  for (int U : {1, 2, 4}) {
    // rows of one workgroup: what U steps of 256 threads cover, at least one; all rows of a position where they fit
    const uint32_t rows = std::max<uint32_t>(1, 256u * U / units);
    const uint32_t tiles_h = (shared + rows - 1) / rows;
    s.h_tile = (shared + tiles_h - 1) / tiles_h;
    s.p_tile = std::max<uint32_t>(1, std::min(s.positions, rows / s.h_tile));
    while (s.p_tile > 1 && s.p_tile * s.angles.pairs > 4096) --s.p_tile;
    const uint32_t h_tiles = (shared + s.h_tile - 1) / s.h_tile, p_tiles = (s.positions + s.p_tile - 1) / s.p_tile;
    s.div_h_tiles = make_fastdiv(h_tiles);
    s.div_inner = make_fastdiv(s.p_inner ? s.p_tile : s.h_tile);
    if (s.div_h_tiles.d == 0 || s.div_inner.d == 0 || (uint64_t)h_tiles * p_tiles >= (1ull << 24)) continue;
    p.iter = U;
    Candidate c = make_candidate(g, "rotary", FS_SCHEME_LDS, K_ROTARY);
    Launch& l = c.launches.front();
    l.args.u.rotary = p;
    l.ptr[0] = in_ref(g, r[0].in);
    if (tensors == 2) l.ptr[1] = in_ref(g, r[1].in);
    l.ptr[2] = in_ref(g, t_pos);
    l.ptr[3] = out_ref(g.tensors[r[0].out].output_slot);
    if (tensors == 2) l.ptr[4] = out_ref(g.tensors[r[1].out].output_slot);
    l.shape.block[0] = 256;
    l.shape.grid[0] = h_tiles * p_tiles;
    l.shape.lds_bytes = s.p_tile * s.angles.pairs * 8;
    c.info.lanes_per_row = (int32_t)std::min<uint32_t>(units, 256);
    c.info.vecs_per_lane = U;
    c.info.rows_per_block = (int32_t)(s.p_tile * s.h_tile);
    c.info.lds_bytes = (int32_t)l.shape.lds_bytes;
    KernelCost kc;
    kc.waves_per_block = 4;
    kc.waves = (double)l.shape.grid[0] * 4;
    kc.lds_bytes_per_block = c.info.lds_bytes;
    kc.vgpr_estimate = 40 + 16 * U;
    const double groups = (double)l.shape.grid[0];
    const double used = n / vec / (p.interleaved && vec > 1 ? 1.0 : 2.0) / (groups * 256.0 * U);   // of the lanes' steps
    const double angles = std::max(1.0, std::ceil(s.p_tile * s.angles.pairs / 256.0));
    kc.own_estimate_s = (3.2 + 0.1 * U + std::max(2.0 * n * esz / 6.2e6 * (1.0 + 0.15 * (1.0 / std::max(0.05, std::min(1.0, used)) - 1.0)),
                                                  groups / 2048.0 * (0.6 * angles + 0.3 * U))) * 1e-6;
    char var[48];
    snprintf(var, sizeof var, "<%s,%s,v%d,U%d,P%u,H%u>", dtype_name(p.in_dt), p.interleaved ? "interleaved" : "halves", p.vec, U, s.p_tile, s.h_tile);
    finish_candidate(&c, var, kc);
    out->push_back(c);
  }
  return true;
}

}  // namespace fs
