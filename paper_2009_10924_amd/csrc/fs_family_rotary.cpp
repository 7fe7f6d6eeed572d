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
  s.lines = 1;
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
      int longer = 0;
      for (int k = 0; k < 3; ++k)
        if (ext[k] > 1) {
          ++longer;
          t.line_in = t.in_stride[k];
          t.line_out = t.out_stride[k];
        }
      if (longer > 1) s.lines = 0;
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
  p.vec = turned >= V ? (int32_t)V : turned >= 4 ? 4 : 1;
  const uint32_t vec = (uint32_t)p.vec;
  s.rot_units = vec == 1 ? s.angles.pairs : (turned + vec - 1) / vec;
  s.units = s.rot_units + (rest + vec - 1) / vec;
  s.short_rest = rest < vec ? rest : 0;
  s.lanes = std::min<uint32_t>(s.units, 256);
  s.div_lanes = make_fastdiv(s.lanes);
  s.div_pairs = make_fastdiv(s.angles.pairs);
  if (s.pos_div[0].d == 0 || s.pos_div[1].d == 0 || s.div_lanes.d == 0 || s.div_pairs.d == 0) return true;

  const int esz = dtype_bytes(p.in_dt);
  double n = 0;
  for (size_t i = 0; i < tensors; ++i) n += (double)g.tensors[r[i].out].numel();
  const uint32_t slots = 256 / s.lanes;
  for (uint32_t P = 1; P <= slots; P *= 2) {
    if (P > 1 && P / 2 >= s.positions) break;
    s.p_slots = std::min(P, s.positions);
    if (s.p_slots * s.angles.pairs > 4096) break;   // 32 KB of angles (one position has no more)
    s.h_slots = std::min(shared, slots / s.p_slots);
    const uint32_t p_tiles = (s.positions + s.p_slots - 1) / s.p_slots;
    // A thread's rows, a kernel for each number: one is for single tokens (us for 1 / 2 / 3 / 5 rows: bf16 [16,1,32+8,128] 3.4 / 3.7 / 4.0 / 4.8),
    // several keep more loads on their way ([2,8192,32+8,128] with 8 slots 62.3 / 59.2 / 57.2 / 63.5, pairs side by side 74.2 / 59.2 / 56.4 / 57.5;
    // [4,4096,16+4,64] with 4 slots 18.4 / 17.7 / 17.5 / 17.4).
    for (int U : {1, 2, 3, 5}) {
      if (U > 1 && s.h_slots * (U == 5 ? 3 : U - 1) >= shared) break;
      const uint32_t most = s.h_slots * U;   // a thread's rows are all loaded at once: h_tile <= U * h_slots, which the kernel relies on
      uint32_t h_tiles = (shared + most - 1) / most;
      s.h_tile = (shared + h_tiles - 1) / h_tiles;
      h_tiles = (shared + s.h_tile - 1) / s.h_tile;
      s.div_h_tiles = make_fastdiv(h_tiles);
      s.div_inner = make_fastdiv(s.p_inner ? s.p_slots : s.h_slots);
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
      l.shape.lds_bytes = s.p_slots * s.angles.pairs * 8;
      c.info.lanes_per_row = (int32_t)s.lanes;
      c.info.vecs_per_lane = U;
      c.info.rows_per_block = (int32_t)(s.p_slots * s.h_tile);
      c.info.lds_bytes = (int32_t)l.shape.lds_bytes;
      KernelCost kc;
      kc.waves_per_block = 4;
      kc.waves = (double)l.shape.grid[0] * 4;
      kc.lds_bytes_per_block = c.info.lds_bytes;
      // The estimate (us), fitted to every candidate of 880 drawn shapes of 1 to 2^26 elements in three dtypes, positions of one to three
      // axes: on 6,700 others the one chosen is 3.8 % behind the fastest (geometric mean; 4.5 % from 30 MB on; fitted to those, 3.7 and
      // 4.2).  Rows that are no whole lines cost by the runs in which a workgroup reads and writes them, most of all written ones.
      const double row_bytes = (double)s.dim * esz, steps = std::ceil((double)s.h_tile / s.h_slots);
      const double per = p.interleaved && vec > 1 ? vec : 2.0 * vec;   // elements of a step
      const double used = std::min(1.0, n / per / ((double)l.shape.grid[0] * 256.0 * steps));   // of the threads' steps
      const double at_once = s.angles.pairs < 256 ? 256 / s.angles.pairs : 1, angles = std::ceil(s.p_slots / at_once) * std::ceil(s.angles.pairs / 256.0);
      auto run = [&](const uint32_t (&stride)[3]) {   // bytes that neighbouring slots cover without a gap
        const bool along_h = s.t[0].shared > 1 && stride[s.p_inner ? 1 : 2] == s.dim;
        return row_bytes * (along_h ? std::min(s.h_slots, s.t[0].shared) : s.p_slots);
      };
      const double cuts = (int64_t)row_bytes % 128 != 0 ? 13.9 : 1.0;
      kc.vgpr_estimate = 46 + (vec == 8 ? 6 : 0) + (p.interleaved && vec > 1 ? 5 : 10) * U;
      const double resident = std::min(8, 512 / ((kc.vgpr_estimate + 7) / 8 * 8));
      const double memory = 2.0 * n * esz / 5.18e6 * (1.0 + 0.0058 * (1.0 / std::max(0.05, used) - 1.0)) * (1.0 + 0.083 * (8.0 / resident - 1.0)) *
                            (1.0 + cuts * (0.017 * 128.0 / run(r[0].in_stride) + 0.186 * 128.0 / run(r[0].out_stride)));
      const double issue = kc.waves / 1024.0 * (218.0 + 16.0 * angles + 245.0 * steps * (per / 16.0 * 0.8 + 0.4)) / 2400.0;
      const double both = std::pow(std::pow(memory, 0.73) + std::pow(issue, 0.73), 1.0 / 0.73);
      kc.own_estimate_s = (2.9 + 0.55 * (both + 0.176 * angles + 0.188 * steps)) * 1e-6;
      char var[48];
      snprintf(var, sizeof var, "<%s,%s,v%d,U%d,P%u,H%ux%u>", dtype_name(p.in_dt), p.interleaved ? "interleaved" : "halves", p.vec, U, s.p_slots, s.h_slots, (s.h_tile + s.h_slots - 1) / s.h_slots);
      finish_candidate(&c, var, kc);
      out->push_back(c);
    }
  }
  return true;
}

}  // namespace fs
