// Pattern families: group normalisation with an activation (channels last), forward and backward.
#include "fs_stitch_util.hpp"

namespace fs {

namespace {

constexpr int64_t kAlign = 256;
int64_t aligned(int64_t bytes) { return (bytes + kAlign - 1) / kAlign * kAlign; }

// mean (or maximum) over a group's positions and channels: axes 1 and 3 of [batch, positions, groups, dim], in either order
bool match_over_group(const fs_graph& g, const char* op, const std::string& inner, int32_t t, MatchState* st) {
  for (const char* axes : {"[-3]|[-1]", "[-1]|[-3]"}) {
    const std::string a(axes, 4), b(axes + 5, 4);
    if (Pattern(std::string(op) + a + "(" + op + b + "(" + inner + "))").match(g, t, st)) return true;
  }
  return false;
}

bool per_group(const Tensor& t, const Tensor& x) {
  return t.rank == 4 && t.dims[0] == x.dims[0] && t.dims[1] == 1 && t.dims[2] == x.dims[2] && t.dims[3] == 1 && t.dtype == FS_F32;
}
bool per_channel(const Tensor& t, const Tensor& x) { return t.numel() == x.dims[2] * x.dims[3] && is_trailing(t, x); }
// gamma and (if there is one) beta: both of x's type, or both float32
bool params_of(const Tensor& gamma, const Tensor* beta, const Tensor& x, GroupNormP* p) {
  if (!per_channel(gamma, x) || (beta && (!per_channel(*beta, x) || beta->dtype != gamma.dtype))) return false;
  p->wide_params = gamma.dtype != x.dtype ? 1 : 0;
  return gamma.dtype == x.dtype || gamma.dtype == FS_F32;
}

bool shape_of(const Tensor& x, GroupNormP* p) {
  p->batch = (uint32_t)x.dims[0];
  p->positions = (uint32_t)x.dims[1];
  p->groups = (uint32_t)x.dims[2];
  p->dim = (uint32_t)x.dims[3];
  p->channels = p->groups * p->dim;
  p->div_dim = make_fastdiv(p->dim);
  p->inv_count = (float)(1.0 / ((double)p->positions * p->dim));
  return p->div_dim.d != 0;
}

// A workgroup of `threads` on sets of `set_groups` groups; false: a position of a set has more vectors than threads, or a
// constant that the kernels need does not exist.
bool lay_out(GroupNormP* p, int threads, uint32_t set_groups) {
  const uint32_t width = set_groups * p->dim;
  p->threads = threads;
  p->set_groups = set_groups;
  p->sets = p->groups / set_groups;
  p->vec = width >= (uint32_t)vec_of(p->dt) ? vec_of(p->dt) : 1;
  p->whole = p->dim % p->vec == 0 ? 1 : 0;
  // Stored past the caches, pieces that share 64 bytes with another workgroup's go to memory one by one: bf16 [8, 4096, 320] in
  // pieces of 20 bytes took 68 us, 33 through the caches; f32 [4, 1024, 512] in pieces of 64 bytes 6.7 past them, 7.4 through.  q's
  // pieces of one byte per value go the same way: by a rule of their own size they are level (f32 [4, 1024, 512] in sets of 16
  // channels 8.48 / 8.48, [16, 256, 1536] in sets of 96 13.25 / 13.27, bf16 [8, 1024, 1024] in sets of 32 14.03 / 14.03).
  p->whole_lines = p->sets == 1 || width * dtype_bytes(p->dt) % 64 == 0 ? 1 : 0;
  p->set_vecs = (width + p->vec - 1) / p->vec;
  if (p->set_vecs > (uint32_t)threads) return false;
  p->rows_at_once = (uint32_t)threads / p->set_vecs;
  p->set_vecs_m = ((1u << 20) + p->set_vecs - 1) / p->set_vecs;
  p->div_per = make_fastdiv(p->whole ? p->dim / p->vec : p->dim);
  p->div_sets = make_fastdiv(p->sets);
  p->div_chunks = make_fastdiv(1);
  p->chunks = 1;
  p->chunk_rows = p->positions;
  p->entries = 1;
  p->entry_blocks = p->batch;
  return p->div_per.d != 0 && p->div_sets.d != 0;
}
int pow2_at_most_log2(uint32_t v) {
  int l = 0;
  while ((2u << l) <= v) ++l;
  return l;
}
// lanes that fold `each` of n sums of `items` values: all threads busy, at most a wavefront, no more lanes than items
int fold_lanes_log2(uint32_t threads, uint32_t n, uint32_t items) {
  return std::min({pow2_at_most_log2(std::max<uint32_t>(1, threads / std::max<uint32_t>(1, n))), 6, log2_of(pow2_at_least(items))});
}
// Chunks of positions for launches of 256 threads: about `want` workgroups in all, each with whole rounds of four positions
// per thread where there are that many.
bool cut(GroupNormP* p, uint32_t want) {
  const uint32_t round = 4 * p->rows_at_once;
  const uint32_t most = std::max<uint32_t>(1, want / (p->batch * p->sets));
  uint32_t rows = std::min((p->positions + most - 1) / most, kGnMostRows * p->rows_at_once);
  rows = std::min(p->positions, (rows + round - 1) / round * round);
  p->chunk_rows = rows;
  p->chunks = (p->positions + rows - 1) / rows;
  p->div_chunks = make_fastdiv(p->chunks);
  return p->div_chunks.d != 0 && (uint64_t)p->batch * p->chunks * p->sets < (1ull << 31);
}
// words of LDS that the items of a position's channels take (gn_pitch)
uint32_t item_pitch(const GroupNormP& p) {
  const uint32_t width = p.set_groups * p.dim;
  return width + (p.vec > 1 ? width / p.vec : 0);
}
// sets of 1 group, of more by twos, of all
std::vector<uint32_t> set_sizes(uint32_t groups) {
  std::vector<uint32_t> s;
  for (uint32_t k = 1; k < groups; k *= 2)
    if (groups % k == 0) s.push_back(k);
  s.push_back(groups);
  return s;
}
// Sets for the launches that read chunk by chunk: the largest whose positions 256 threads cover, and, where its pieces are whole
// 64-byte pieces of memory, the smallest of at least 512 bytes of a position: more positions per workgroup, so fewer chunks whose
// partial results are written and read (f16 [1, 2295, 1664] backward: sums as large as the values otherwise).
std::vector<uint32_t> chunk_sets(const GroupNormP& p) {
  std::vector<uint32_t> sets;
  uint32_t narrow = 0;
  for (uint32_t s = std::min(p.groups, 256u * 8); s >= 1; --s) {   // (a thread has at most 8 values of a position)
    GroupNormP q = p;
    if (p.groups % s != 0 || !lay_out(&q, 256, s)) continue;
    if (sets.empty()) sets.push_back(s);
    const uint32_t bytes = s * p.dim * (uint32_t)dtype_bytes(p.dt);
    if (bytes >= 512 && bytes % 64 == 0) narrow = s;
  }
  if (narrow && narrow != sets[0]) sets.push_back(narrow);
  return sets;
}

// Whether the last launch's workgroups join their groups' chunks themselves: a launch less, where one batch of `loads` loads per
// lane brings all of them (a second one costs more than a launch).
bool joins(const GroupNormP& p, uint32_t set_groups, uint32_t loads) {
  return (uint64_t)p.chunks * std::max<uint32_t>(set_groups, 4) <= 256ull * loads;
}

// What the launches read and write, and the estimate of their time.  These kernels are short: most of what a shape costs is the
// chain of instructions of one wavefront (which hardly any other covers) against its share of the arithmetic and the bytes, which
// the general evaluator has no terms for.  Constants fitted to every candidate of 700 shapes of 1 to 2^26 elements, three dtypes, timed
// on three sets of buffers in turn; the candidate chosen was 2.2 % behind the fastest (geometric mean of 500 further shapes; 2.5 %
// forward and 3.0 % backward on 140 drawn later), 12 % by the general evaluator.
struct Traffic {
  double read_bytes = 0, written_bytes = 0, act = 0;   // act: 0 none, 1 SiLU, 1.5 tanh-GELU
  bool backward = false;
};
struct SlabModel { double ops, ops_act, ops_8bit, fixed, chain_op, chain_item, chain_threads, issue, issue_op, shared_lines, overlap, fold, line, round; };
const SlabModel kSlab[2] = {{4.92, 4.92, 3.24, 3.07, 1.94e-3, 0.131, 0.0, 0.682, 4.5e-4, 0.125, 0.0, 0.0, 9.6e-4, 0.652},
                            {1.87, 8.05, 0.02, 3.47, 6.0e-3, 0.057, 0.047, 0.887, 0.0, 0.107, 0.0054, 2.66, 1.2e-4, 1.175}};
struct PassesModel { double ops, ops_act, ops_8bit, issue_op, reread_l2, reread, fixed, launch, overlap, item, partials, join, shared_lines; };
const PassesModel kPasses[2] = {{7.95, 4.93, 5.02, 3.42e-3, 0.68, 0.73, 6.71, 2.47, 0.018, 0.192, 0.0, 1.87e-4, 0.24},
                                {7.99, 5.02, 4.90, 4.9e-3, 0.63, 0.64, 6.86, 2.48, 0.309, 0.273, 1.1, 2.02e-4, 0.15}};
// items that a lane adds up of what a workgroup's threads have gathered: a group's (forward), a channel's (backward)
double items_per_lane(const GroupNormP& p, bool backward) {
  const double per = backward ? p.rows_at_once : (p.whole ? (double)p.dim / p.vec : (double)p.dim) * p.rows_at_once;
  const double sums = backward ? (double)p.set_groups * p.dim : p.set_groups;
  const double lanes = std::max(1.0, std::min(64.0, std::floor(p.threads / sums)));
  return per / lanes * std::max(1.0, sums / p.threads);
}
// what `workgroups` of them stream at most, each on a compute unit of its own
double few_units(double bytes, double workgroups, double unit) { return bytes / std::min(256.0, workgroups) / unit; }
double slab_us(const GroupNormP& p, const Traffic& t, int esz, int K, int vgprs) {
  const SlabModel& m = kSlab[t.backward ? 1 : 0];
  const double groups = (double)p.entry_blocks * p.sets;
  const double waves = std::max(1.0, groups * p.threads / 64.0 / 1024.0);   // per SIMD
  const double ops = (m.ops + m.ops_act * t.act + m.ops_8bit * p.checkpoint) * K * p.vec;
  // workgroups that a compute unit holds, and so the rounds of them
  const int per_simd = std::min(8, 512 / std::max(8, (vgprs + 7) / 8 * 8)), held = std::max(1, 4 * per_simd / (p.threads / 64));
  const double rounds = std::min(8.0, std::ceil(groups / (256.0 * held)));
  const double chain = (m.fixed + m.chain_op * ops + m.chain_item * items_per_lane(p, t.backward) + m.chain_threads * p.threads / 512.0) * (1.0 + m.round * (rounds - 1.0));
  if (p.entries > 1 && p.entry_blocks == 1) {   // a few entries after one another and no other launch (fitted to 420 such candidates, 7 % rms)
    const double sums_per_lane = p.dim / std::max(1.0, std::min(64.0, std::floor((double)p.threads / p.set_groups)));
    const double each = 0.61 + 6.0e-3 * ops + 0.094 * items_per_lane(p, true) + 0.71 * p.threads / 512.0 + 0.21 * sums_per_lane;
    return 2.89 + std::max(each * p.entries, few_units(t.read_bytes + t.written_bytes, groups, 3.3e4));
  }
  const double more = std::max(0.0, chain - 1.5) * (p.entries - 1.0);   // the next entries' chains, without a launch
  const double issue = waves * (m.issue + m.issue_op * ops);
  const double run = p.sets > 1 ? (double)p.set_groups * p.dim * esz : 1e9;
  double memory = (t.read_bytes + t.written_bytes) / 6.5e6 * (1.0 + m.shared_lines * std::max(0.0, 256.0 / run - 1.0));
  memory = std::max(memory, few_units(t.read_bytes + t.written_bytes, groups, 3.3e4));
  // lines that the accesses of a compute unit's wavefronts touch, one after the other
  memory = std::max(memory, m.line * K * p.threads / 64.0 * std::max(1.0, groups / 256.0) * std::max(64.0 / p.set_vecs, 64.0 * p.vec * esz / 128.0));
  if (t.backward && p.entry_blocks > 1) memory += 16.0 * p.entry_blocks * p.channels / 6.6e6;   // partial sums, written and read
  return chain + more + std::max(issue, memory) + m.overlap * std::min(issue, memory) + (p.entry_blocks > 1 ? m.fold : 0.0);
}
double passes_us(const GroupNormP& p, const Traffic& t, size_t n_launches) {
  const PassesModel& m = kPasses[t.backward ? 1 : 0];
  const double waves = std::max(1.0, (double)p.batch * p.sets * p.chunks * 4.0 / 1024.0);
  const double rows = std::ceil((double)p.chunk_rows / p.rows_at_once);
  const double issue = waves * rows * p.vec * (m.ops + m.ops_act * t.act + m.ops_8bit * p.checkpoint) * m.issue_op;
  const double again = t.read_bytes < 2.4e7 ? m.reread_l2 : t.read_bytes < 2e8 ? m.reread : 1.0;   // from the dies' caches, the memory-side one
  double memory = t.read_bytes / 6.8e6 + (t.read_bytes * again + t.written_bytes) / 6.6e6 +
                  m.partials * 16.0 * p.batch * p.chunks * p.channels / 6.6e6 + m.join * p.chunks * p.set_groups;
  if (p.sets > 1) memory *= 1.0 + m.shared_lines * 128.0 / ((double)p.set_groups * p.dim * dtype_bytes(p.dt));
  const double workgroups = (double)p.batch * p.sets * p.chunks;
  // very many short workgroups: their prologues, in both launches; and the second one of a compute unit, whose gathering ends when
  // the first one's does (twice the workgroups are 5 % slower in calls of 12 us and 8 % faster in those of 50)
  const double starts = 1.1 * std::max(0.0, waves - 2.0) + (workgroups > 256.0 ? 1.1 : 0.0);
  if (workgroups < 400) memory *= 1.05;   // one wavefront per SIMD: loads and arithmetic take turns
  memory = std::max(memory, few_units(2.0 * t.read_bytes + t.written_bytes, workgroups, 4.0e4));
  return m.fixed + m.launch * ((double)n_launches - 2.0) + starts + std::max(issue, memory) + m.overlap * std::min(issue, memory) + m.item * items_per_lane(p, t.backward);
}
KernelCost estimated(double us, const GroupNormP& p, int vgprs, int lds) {
  KernelCost kc;
  kc.own_estimate_s = us * 1e-6;
  kc.vgpr_estimate = vgprs;
  kc.waves_per_block = p.threads / 64;
  kc.lds_bytes_per_block = lds;
  return kc;
}

}  // namespace

// ------------------------------------------------------------------ forward
bool build_group_norm(const fs_graph& g, std::vector<Candidate>* out, PackForm*) {
  if (g.outputs.empty() || g.outputs.size() > 5 || g.inputs.size() != 3 || g.tensors[g.inputs[0]].rank > 4) return false;
  MatchState st;
  int32_t t_q = -1, t_s = -1, t_y = -1, act = ACT_NONE;
  bool has_8bit = false;
  for (int32_t t : g.outputs) has_8bit = has_8bit || g.tensors[t].store_as == FS_E4M3;
  if (has_8bit && !match_8bit(g, "rmax[-3](rmax[-1](abs($V)))", &st, &t_q, &t_s) && !match_8bit(g, "rmax[-1](rmax[-3](abs($V)))", &st, &t_q, &t_s))
    return false;
  for (int32_t t : g.outputs)
    if (t != t_q && (t_y < 0 || g.tensors[t].numel() > g.tensors[t_y].numel())) t_y = t;
  if (t_y < 0 || g.tensors[t_y].rank != 4) return false;
  MatchState with_act = st;
  if (match_activation(g, t_y, &with_act, &act)) st = with_act;
  else st.tensors["Z"] = t_y;
  const char* affine = "add(mul(mul(sub($X,$MU),rsqrt(addc[#0]($VAR))),$G),$B)";
  if (!Pattern(affine).match(g, st.tensors["Z"], &st)) return false;
  // (the same ops once more, to know the normalised values' tensor)
  if (!Pattern("add(mul($N,$G),$B)").match(g, st.tensors["Z"], &st) || !Pattern("mul($C,rsqrt(addc[#0]($VAR)))").match(g, st.tensors["N"], &st)) return false;
  if (has_8bit && st.tensors["V"] != st.tensors["N"]) return false;
  if (!match_over_group(g, "rmean", "square($C)", st.tensors["VAR"], &st) || !match_over_group(g, "rmean", "$X", st.tensors["MU"], &st)) return false;
  if (!covers_all(g, st)) return false;
  const int32_t tx = st.tensors["X"], tg = st.tensors["G"], tb = st.tensors["B"];
  for (int32_t t : {tx, tg, tb})
    if (!is_input(g, t)) return false;
  int32_t t_mu = -1, t_r = -1;
  for (int32_t t : g.outputs) {
    if (t == t_y || t == t_q || t == t_s) continue;
    if (g.tensors[t].store_as != FS_F32) return true;
    const int32_t opcode = g.ops[g.tensors[t].producer].opcode;
    if (t == st.tensors["MU"]) t_mu = t;
    else if (opcode == FS_RSQRT) t_r = t;
    else return true;
  }
  const Tensor& x = g.tensors[tx];
  GroupNormP base{};
  base.dt = x.dtype;
  base.act = act;
  base.checkpoint = has_8bit ? 1 : 0;
  if (x.rank != 4 || !is_float_dtype(x.dtype) || !same_dims(x, g.tensors[t_y]) || g.tensors[t_y].store_as != x.dtype ||
      !params_of(g.tensors[tg], &g.tensors[tb], x, &base) || !shape_of(x, &base))
    return true;
  base.eps = (float)st.scalars[0];
  if (has_8bit) {
    // values become 8 bits by one factor, rstd / scale: finite for groups of equal values too
    if (!(st.scalars[0] > 0.0 && 1.0 / (std::sqrt(st.scalars[0]) * st.scalars[81]) < 1e38)) return true;
    base.inv_max = (float)st.scalars[80];
    base.tiny = (float)st.scalars[81];
  }
  const int esz = dtype_bytes(base.dt);
  Traffic t;
  t.read_bytes = (double)x.numel() * esz;
  t.written_bytes = (double)x.numel() * (esz + (has_8bit ? 1 : 0));
  t.act = act == ACT_GELU ? 1.5 : act == ACT_SILU ? 1.0 : 0.0;

  // ---- one launch
  struct Slab { int threads, K; };
  for (uint32_t gs : set_sizes(base.groups)) {
    for (Slab sh : {Slab{64, 1}, Slab{64, 2}, Slab{64, 4}, Slab{256, 1}, Slab{256, 2}, Slab{256, 4}, Slab{256, 8}, Slab{512, 4}, Slab{512, 8}, Slab{512, 16}, Slab{512, 32}}) {
      GroupNormP p = base;
      if (!lay_out(&p, sh.threads, gs)) continue;
      const uint64_t held = (uint64_t)sh.K * p.rows_at_once;
      if (held < p.positions || (sh.K > 1 && held >= 2ull * p.positions + p.rows_at_once)) continue;
      if (held * p.channels * esz >= (1ull << 32)) continue;   // the kernel's distances within a batch entry
      const uint32_t items = p.rows_at_once * (p.whole ? p.set_vecs : item_pitch(p));
      p.vecs_per_lane = sh.K;
      p.fold_log2 = fold_lanes_log2(sh.threads, gs, p.rows_at_once * (p.whole ? p.dim / p.vec : p.dim));
      const int64_t lds = 4ll * ((has_8bit ? 2 : 1) * (int64_t)items + 3 * gs);
      if (lds > 64 * 1024 || (uint64_t)p.batch * p.sets >= (1ull << 31)) continue;
      Candidate c = make_candidate(g, "group_norm", FS_SCHEME_LDS, K_GN_SLAB);
      Launch& l = c.launches.front();
      l.args.u.gn = p;
      l.ptr[0] = in_ref(g, tx);
      l.ptr[1] = in_ref(g, tg);
      l.ptr[2] = in_ref(g, tb);
      l.ptr[3] = out_ref(g.tensors[t_y].output_slot);
      if (t_mu >= 0) l.ptr[4] = out_ref(g.tensors[t_mu].output_slot);
      if (t_r >= 0) l.ptr[5] = out_ref(g.tensors[t_r].output_slot);
      if (t_q >= 0) { l.ptr[6] = out_ref(g.tensors[t_q].output_slot); l.ptr[7] = out_ref(g.tensors[t_s].output_slot); }
      l.shape.block[0] = (uint32_t)sh.threads;
      l.shape.grid[0] = p.batch * p.sets;
      l.shape.lds_bytes = (uint32_t)lds;
      c.info.lanes_per_row = (int32_t)p.set_vecs;
      c.info.vecs_per_lane = sh.K;
      c.info.rows_per_block = (int32_t)p.rows_at_once;
      c.info.lds_bytes = (int32_t)lds;
      const int vgprs = 40 + sh.K * (p.vec * esz / 4 + 1);
      const KernelCost kc = estimated(slab_us(p, t, esz, sh.K, vgprs), p, vgprs, (int)lds);
      char var[56];
      snprintf(var, sizeof var, "<%s,%s,T%d,K%d,G%u>", dtype_name(p.dt), act_name(act), sh.threads, sh.K, gs);
      finish_candidate(&c, var, kc);
      out->push_back(c);
    }
  }

  // ---- two or three launches
  for (uint32_t gs : chunk_sets(base)) {
    uint32_t last_chunks = 0;
    for (uint32_t want : {256u, 512u}) {
      GroupNormP p = base;
      if (!lay_out(&p, 256, gs) || !cut(&p, want) || p.chunks == last_chunks) continue;
      last_chunks = p.chunks;
      const uint32_t items = p.rows_at_once * (p.whole ? p.set_vecs : item_pitch(p));
      const int64_t lds = 4ll * ((has_8bit ? 4 : 2) * (int64_t)items + p.rows_at_once);
      const int64_t chunk_bytes = aligned((has_8bit ? 16ll : 8ll) * p.batch * p.chunks * p.groups);
      const bool join = joins(p, gs, has_8bit ? 8 : 16);
      Candidate c = make_candidate(g, "group_norm", FS_SCHEME_GLOBAL, K_GN_STATS);
      {
        Launch& l = c.launches.front();
        p.fold_log2 = fold_lanes_log2(256, gs, p.rows_at_once * (p.whole ? p.dim / p.vec : p.dim));
        l.args.u.gn = p;
        l.ptr[0] = in_ref(g, tx);
        l.ptr[1] = ws_ref(0);
        l.shape.block[0] = 256;
        l.shape.grid[0] = p.batch * p.chunks * p.sets;
        l.shape.lds_bytes = (uint32_t)lds;
      }
      auto statistics = [&](Launch& l, int first) {
        if (t_mu >= 0) l.ptr[first] = out_ref(g.tensors[t_mu].output_slot);
        if (t_r >= 0) l.ptr[first + 1] = out_ref(g.tensors[t_r].output_slot);
        if (t_s >= 0) l.ptr[first + 2] = out_ref(g.tensors[t_s].output_slot);
      };
      if (!join) {
        c.launches.emplace_back();
        Launch& l = c.launches.back();
        l.kernel = K_GN_JOIN;
        l.args.u.gn = p;
        l.args.u.gn.fold_log2 = std::min(6, log2_of(pow2_at_least(p.chunks)));
        l.ptr[0] = ws_ref(0);
        l.ptr[1] = ws_ref(chunk_bytes);
        statistics(l, 2);
        const uint32_t at_once = 256u >> l.args.u.gn.fold_log2;
        l.shape.block[0] = 256;
        l.shape.grid[0] = (p.batch * p.groups + at_once - 1) / at_once;
      }
      {
        c.launches.emplace_back();
        Launch& l = c.launches.back();
        l.kernel = K_GN_APPLY;
        l.args.u.gn = p;
        l.args.u.gn.join = join ? 1 : 0;
        l.args.u.gn.fold_log2 = fold_lanes_log2(256, gs, p.chunks);
        l.ptr[0] = in_ref(g, tx);
        l.ptr[1] = in_ref(g, tg);
        l.ptr[2] = in_ref(g, tb);
        l.ptr[3] = ws_ref(join ? 0 : chunk_bytes);
        l.ptr[4] = out_ref(g.tensors[t_y].output_slot);
        if (t_q >= 0) l.ptr[5] = out_ref(g.tensors[t_q].output_slot);
        if (join) statistics(l, 6);
        l.shape.block[0] = 256;
        l.shape.grid[0] = p.batch * p.chunks * p.sets;
        l.shape.lds_bytes = join ? 16 * gs : 0;
      }
      c.info.n_kernels = (int32_t)c.launches.size();
      c.info.workspace_bytes = chunk_bytes + (join ? 0 : aligned(16ll * p.batch * p.groups));
      c.info.bytes_moved_model = c.info.bytes_min + (int64_t)t.read_bytes;
      c.info.lanes_per_row = (int32_t)p.set_vecs;
      c.info.vecs_per_lane = 4;
      c.info.rows_per_block = (int32_t)p.chunk_rows;
      c.info.lds_bytes = (int32_t)lds;
      const KernelCost kc = estimated(passes_us(p, t, c.launches.size()), p, 96, (int)lds);
      char var[56];
      snprintf(var, sizeof var, "<%s,%s,G%u,C%u,%sapply>", dtype_name(p.dt), act_name(act), gs, p.chunks, join ? "" : "join,");
      finish_candidate(&c, var, kc);
      out->push_back(c);
    }
  }
  // Very many short groups, one per batch entry: a workgroup each takes 0.31 ns (0.39 with a checkpoint) whatever little it holds, and
  // the ops one by one, whose sums then run along rows, need not take longer (us, kernels / op by op: f32 [2^24, 1, 1] 4919 / 406, [2^20, 1, 4]
  // 350 / 84, [919002, 2, 16] 311 / 348, bf16 [126575, 9, 1] 42 / 51).  With several groups those sum along a middle axis and are slower.
  if (base.groups == 1 && base.batch >= (1u << 16)) {
    Candidate ops;
    if (build_unfused(g, &ops) == FS_OK) {
      predict(&ops);
      if ((has_8bit ? 3.9e-4 : 3.1e-4) * base.batch > 1.25 * ops.info.predicted_us) out->clear();
    }
  }
  return true;
}

// ------------------------------------------------------------------ backward
bool build_group_norm_backward(const fs_graph& g, std::vector<Candidate>* out, PackForm*) {
  if (g.outputs.size() != 3) return false;
  // two sums over batch and positions, and dx
  int32_t t_dx = -1, t_sum[2] = {-1, -1}, of[2] = {-1, -1};
  std::set<int32_t> sum_ops;
  int n_sums = 0;
  for (int32_t t : g.outputs) {
    if (g.tensors[t].rank != 4) return false;
    const Op& op = g.ops[g.tensors[t].producer];
    if (op.opcode != FS_REDUCE_SUM) {
      if (t_dx >= 0) return false;
      t_dx = t;
      continue;
    }
    const Tensor& inner = g.tensors[op.in[0]];
    if (n_sums == 2 || inner.producer < 0 || inner.output_slot >= 0) return false;
    const Op& first = g.ops[inner.producer];
    if (first.opcode != FS_REDUCE_SUM || first.axis + op.axis != 1) return false;   // axes 0 and 1
    sum_ops.insert(g.tensors[t].producer);
    sum_ops.insert(inner.producer);
    t_sum[n_sums] = t;
    of[n_sums++] = first.in[0];
  }
  if (n_sums != 2 || t_dx < 0) return false;
  MatchState st;
  int32_t t_dbeta = -1, t_dgamma = -1;
  for (int k = 0; k < 2 && t_dbeta < 0; ++k) {   // dbeta sums DZ, dgamma DZ times the normalised values
    MatchState trial;
    trial.tensors["DZ"] = of[k];
    if (!Pattern("mul($DZ,$N)").match(g, of[1 - k], &trial)) continue;
    if (!Pattern("mul(sub(sub($GG,$M1),mul($N,$M2)),$R)").match(g, t_dx, &trial)) continue;
    if (!Pattern("mul($DZ,$G)").match(g, trial.tensors["GG"], &trial)) continue;
    if (!match_over_group(g, "rmean", "$GG", trial.tensors["M1"], &trial) || !match_over_group(g, "rmean", "mul($GG,$N)", trial.tensors["M2"], &trial)) continue;
    st = trial;
    t_dbeta = t_sum[k];
    t_dgamma = t_sum[1 - k];
  }
  if (t_dbeta < 0) return false;
  GroupNormP base{};
  base.act = ACT_NONE;
  const int32_t tdz = st.tensors["DZ"], tn = st.tensors["N"];
  int32_t tdy = tdz, tb = -1;
  if (!is_input(g, tdz)) {
    if (!match_activation_gradient(g, tdz, &st, &base.act)) return false;
    tdy = st.tensors["DY"];
    if (!Pattern("add(mul($N,$G),$B)").match(g, st.tensors["Z"], &st)) return false;
    tb = st.tensors["B"];
    if (!is_input(g, tb)) return false;
  }
  int32_t tx, tcentre;
  if (Pattern("mul(sub($X,$MU),$R)").match(g, tn, &st)) {
    tx = st.tensors["X"];
    tcentre = st.tensors["MU"];
  } else {
    if (!Pattern("mul($Q,$S)").match(g, tn, &st)) return false;
    tx = st.tensors["Q"];
    tcentre = st.tensors["S"];
    if (!is_input(g, tx) || !is_input(g, tcentre)) return false;
    if (g.tensors[tx].dtype != FS_E4M3) std::swap(tx, tcentre);
    if (g.tensors[tx].dtype != FS_E4M3) return false;
    base.checkpoint = 1;
  }
  for (int32_t op : sum_ops) st.covered.insert(op);
  if (!covers_all(g, st)) return false;
  const int32_t tr = st.tensors["R"], tg = st.tensors["G"];
  for (int32_t t : {tx, tcentre, tr, tg, tdy})
    if (!is_input(g, t)) return false;
  const Tensor& dy = g.tensors[tdy];
  base.dt = dy.dtype;
  const Tensor& x = g.tensors[tx];
  if (dy.rank != 4 || !is_float_dtype(dy.dtype) || !same_dims(x, dy) || (!base.checkpoint && x.dtype != dy.dtype) || !same_dims(g.tensors[t_dx], dy) ||
      g.tensors[t_dx].store_as != dy.dtype || g.tensors[t_dbeta].store_as != FS_F32 || g.tensors[t_dgamma].store_as != FS_F32 ||
      !per_group(g.tensors[tcentre], dy) || !per_group(g.tensors[tr], dy) || !params_of(g.tensors[tg], tb >= 0 ? &g.tensors[tb] : nullptr, dy, &base) ||
      !shape_of(dy, &base))
    return true;
  const int esz = dtype_bytes(base.dt), xsz = base.checkpoint ? 1 : esz;
  const uint32_t pitch = colsum_pitch(base.channels);
  Traffic t;
  t.read_bytes = (double)dy.numel() * (esz + xsz);
  t.written_bytes = (double)dy.numel() * esz;
  t.act = base.act == ACT_GELU ? 1.5 : base.act == ACT_SILU ? 1.0 : 0.0;
  t.backward = true;
  auto fill_inputs = [&](Launch& l) {
    l.ptr[0] = in_ref(g, tx);
    l.ptr[1] = in_ref(g, tcentre);
    l.ptr[2] = in_ref(g, tr);
    l.ptr[3] = in_ref(g, tg);
    if (tb >= 0) l.ptr[4] = in_ref(g, tb);
    l.ptr[5] = in_ref(g, tdy);
  };
  // ---- one launch and the fold
  struct Slab { int threads, K; };
  for (uint32_t gs : set_sizes(base.groups)) {
    for (Slab sh : {Slab{64, 1}, Slab{64, 2}, Slab{64, 4}, Slab{256, 1}, Slab{256, 2}, Slab{256, 4}, Slab{512, 4}, Slab{512, 8}, Slab{512, 16}}) {
      GroupNormP p = base;
      if (!lay_out(&p, sh.threads, gs)) continue;
      const uint64_t held = (uint64_t)sh.K * p.rows_at_once;
      if (held < p.positions || (sh.K > 1 && held >= 2ull * p.positions + p.rows_at_once)) continue;
      if (held * p.channels * esz >= (1ull << 32)) continue;
      const uint32_t width = gs * p.dim;
      p.vecs_per_lane = sh.K;
      p.fold_log2 = fold_lanes_log2(sh.threads, width, p.rows_at_once);
      p.means_log2 = fold_lanes_log2(sh.threads, gs, p.dim);
      // One batch entry per workgroup; of very many entries so many that the partial sums stay small beside the values (f16
      // [65536, 1, 512]: 268 MB of them beside 200 MB otherwise); or, of two to four, all: their sums are complete, a launch less
      // (bf16 [2, 16, 256] 7.8 -> 6.6 us, [3, 1, 128] 7.7 -> 5.4, [8, 1, 128] no faster).
      const uint32_t most = std::max<uint32_t>(1, 8192 / p.sets);
      const uint32_t many = p.batch > most && sh.threads <= 256 ? (p.batch + most / 4 - 1) / std::max<uint32_t>(1, most / 4) : 1;
      std::vector<uint32_t> entries = {many};
      if (p.batch > 1 && p.batch <= 4 && sh.threads <= 256) entries.push_back(p.batch);
      for (uint32_t e : entries) {
        p.entries = e;
        p.entry_blocks = (p.batch + e - 1) / e;
        const bool fold = p.entry_blocks > 1;
        const int64_t sum_bytes = aligned(8ll * p.entry_blocks * pitch);
        const int64_t lds = 4ll * (2ll * p.rows_at_once * item_pitch(p) + 3 * width + 2 * gs + (e > 1 ? 2 * width : 0));
        if (lds > 64 * 1024 || (uint64_t)p.entry_blocks * p.sets >= (1ull << 31)) continue;
        Candidate c = make_candidate(g, "group_norm_backward", FS_SCHEME_LDS, K_GN_BWD_SLAB);
        Launch& l = c.launches.front();
        l.args.u.gn = p;
        fill_inputs(l);
        l.ptr[6] = out_ref(g.tensors[t_dx].output_slot);
        l.ptr[7] = fold ? ws_ref(0) : out_ref(g.tensors[t_dbeta].output_slot);
        l.ptr[8] = fold ? ws_ref(4ll * pitch) : out_ref(g.tensors[t_dgamma].output_slot);
        l.shape.block[0] = (uint32_t)sh.threads;
        l.shape.grid[0] = p.entry_blocks * p.sets;
        l.shape.lds_bytes = (uint32_t)lds;
        const int vgprs = 73 + sh.K * (p.vec * (esz + xsz) / 4 + 1);
        const KernelCost kc = estimated(slab_us(p, t, esz, sh.K, vgprs), p, vgprs, (int)lds);
        char var[56];
        snprintf(var, sizeof var, "<%s,%s,T%d,K%d,G%u,E%u%s>", dtype_name(p.dt), act_name(p.act), sh.threads, sh.K, gs, e, fold ? ",fold" : "");
        finish_candidate(&c, var, kc);
        if (fold) {   // dbeta from the first half of each row of sums, dgamma from the second
          c.launches.emplace_back();
          Launch& f = c.launches.back();
          make_fold_launch(&f, p.entry_blocks, 2 * pitch, pitch, p.channels);
          f.ptr[0] = ws_ref(0);
          f.ptr[1] = out_ref(g.tensors[t_dbeta].output_slot);
          f.ptr[2] = out_ref(g.tensors[t_dgamma].output_slot);
          c.info.n_kernels = 2;
          c.info.workspace_bytes = sum_bytes;
          c.info.bytes_moved_model = c.info.bytes_min + 2 * sum_bytes;
        }
        c.info.lanes_per_row = (int32_t)p.set_vecs;
        c.info.vecs_per_lane = sh.K;
        c.info.rows_per_block = (int32_t)p.rows_at_once;
        c.info.lds_bytes = (int32_t)lds;
        out->push_back(c);
      }
    }
  }

  // ---- two or three launches
  for (uint32_t gs : chunk_sets(base)) {
    uint32_t last_chunks = 0;
    for (uint32_t want : {256u, 512u}) {
      GroupNormP p = base;
      if (!lay_out(&p, 256, gs) || !cut(&p, want) || p.chunks == last_chunks) continue;
      last_chunks = p.chunks;
      const uint32_t width = gs * p.dim, rows = p.batch * p.chunks;
      const int64_t lds = 4ll * (2ll * p.rows_at_once * item_pitch(p) + 3 * width);
      const int64_t chunk_bytes = aligned(8ll * rows * pitch), mean_bytes = aligned(8ll * rows * p.groups);
      const bool join = joins(p, gs, 16);
      Candidate c = make_candidate(g, "group_norm_backward", FS_SCHEME_GLOBAL, K_GN_BWD_SUMS);
      {
        Launch& l = c.launches.front();
        p.fold_log2 = fold_lanes_log2(256, width, p.rows_at_once);
        p.means_log2 = fold_lanes_log2(256, gs, p.dim);
        l.args.u.gn = p;
        fill_inputs(l);
        l.ptr[6] = ws_ref(0);
        l.ptr[7] = ws_ref(chunk_bytes);
        l.shape.block[0] = 256;
        l.shape.grid[0] = rows * p.sets;
        l.shape.lds_bytes = (uint32_t)lds;
      }
      if (!join) {
        c.launches.emplace_back();
        Launch& l = c.launches.back();
        l.kernel = K_GN_BWD_JOIN;
        l.args.u.gn = p;
        l.args.u.gn.fold_log2 = std::min(6, log2_of(pow2_at_least(p.chunks)));
        l.ptr[0] = ws_ref(chunk_bytes);
        l.ptr[1] = ws_ref(chunk_bytes + mean_bytes);
        const uint32_t at_once = 256u >> l.args.u.gn.fold_log2;
        l.shape.block[0] = 256;
        l.shape.grid[0] = (p.batch * p.groups + at_once - 1) / at_once;
      }
      {
        c.launches.emplace_back();
        Launch& l = c.launches.back();
        l.kernel = K_GN_BWD_APPLY;
        GroupNormP& q = l.args.u.gn;
        q = p;
        q.join = join ? 1 : 0;
        q.fold_log2 = fold_lanes_log2(256, gs, p.chunks);
        const uint32_t quads = rows > 128 ? 4 : 16;   // quads of columns per workgroup of the fold
        q.fold_blocks = ((2 * pitch / 4 + quads - 1) / quads + 7) / 8 * 8;
        fill_inputs(l);
        l.ptr[6] = out_ref(g.tensors[t_dx].output_slot);
        l.ptr[7] = ws_ref(join ? chunk_bytes : chunk_bytes + mean_bytes);
        l.ptr[8] = ws_ref(0);
        l.ptr[9] = out_ref(g.tensors[t_dbeta].output_slot);
        l.ptr[10] = out_ref(g.tensors[t_dgamma].output_slot);
        l.shape.block[0] = 256;
        l.shape.grid[0] = q.fold_blocks + rows * p.sets;
        l.shape.lds_bytes = std::max<uint32_t>(4096, join ? 8 * gs : 0);
      }
      c.info.n_kernels = (int32_t)c.launches.size();
      c.info.workspace_bytes = chunk_bytes + mean_bytes + (join ? 0 : aligned(8ll * p.batch * p.groups));
      c.info.bytes_moved_model = c.info.bytes_min + (int64_t)t.read_bytes + 2 * chunk_bytes;
      c.info.lanes_per_row = (int32_t)p.set_vecs;
      c.info.vecs_per_lane = 4;
      c.info.rows_per_block = (int32_t)p.chunk_rows;
      c.info.lds_bytes = (int32_t)lds;
      const KernelCost kc = estimated(passes_us(p, t, c.launches.size()), p, 120, (int)lds);
      char var[56];
      snprintf(var, sizeof var, "<%s,%s,G%u,C%u,%sapply>", dtype_name(p.dt), act_name(p.act), gs, p.chunks, join ? "" : "join,");
      finish_candidate(&c, var, kc);
      out->push_back(c);
    }
  }
  return true;
}

}  // namespace fs
