"""How many additions in a row a sum of the group normalisation and checkpoint kernels takes, from the launch shapes that plans choose
from: the bounds of the GPU tests count 100 of them, which is a property of the shapes listed there (a thread may have 128
positions, a workgroup any number of batch entries).  No GPU."""
import re

import pytest

from paper_2009_10924_amd import binding as B
from workloads import checkpoint_backward_graph, group_norm_backward_graph, group_norm_graph

from . import test_gpu_checkpoint, test_gpu_group_norm

TREE = 6                      # steps of a sum over a wavefront's lanes
ceil = lambda a, b: -(-a // b)   # noqa: E731


def pow2_at_most(v):
    return 1 << (max(1, v).bit_length() - 1)


def pow2_at_least(v):
    return 1 << (max(1, v) - 1).bit_length()


def fold_lanes(threads, sums, items):
    return min(pow2_at_most(threads // max(1, sums)), 64, pow2_at_least(items))


def folded_rows(rows):
    """K_COLFOLD: 64 or 16 row groups, then three or two levels of four."""
    return 0 if rows <= 1 else ceil(rows, 64) + 9 if rows > 128 else ceil(rows, 16) + 6


def group_norm_chain(info, shape, dtype, backward):
    """Longest chain of additions of a candidate."""
    batch, positions, groups, dim = shape
    elems = 4 if dtype == "f32" else 8
    tag = re.match(r"gn_(?:bwd_)?(slab|stats|sums)<\w+,\w+,(.*)>", info["kernel"]).groups()
    field = {k: int(v) for k, v in re.findall(r"([TKGEC])(\d+)", tag[1])}
    threads, gs = field.get("T", 256), field["G"]
    width = gs * dim
    vec = elems if width >= elems else 1
    whole = dim % vec == 0
    set_vecs = ceil(width, vec)
    rows = threads // set_vecs
    per = dim // vec if whole else dim
    slab = tag[0] == "slab"
    own = field["K"] if slab else ceil(info["rows_per_block"], rows)
    if backward:
        channel = own + ceil(rows, fold_lanes(threads, width, rows)) + TREE
        group = channel + ceil(dim, fold_lanes(threads, gs, dim)) + TREE
        if slab:
            entries = field["E"]
            return max(group, channel + entries + folded_rows(ceil(batch, entries)))
        chunks = field["C"]
        # every workgroup of the last launch joins them, or a launch of its own does, each group's by as many lanes as there are chunks
        joined = ceil(chunks, min(64, pow2_at_least(chunks)) if "join" in info["kernel"] else fold_lanes(256, gs, chunks)) + TREE
        return max(group + joined, channel + folded_rows(batch * chunks))
    chain = own + (vec if whole else 0) + ceil(rows * per, fold_lanes(threads, gs, rows * per)) + TREE
    if not slab:
        chunks = field["C"]
        lanes = min(64, pow2_at_least(chunks)) if "join" in info["kernel"] else fold_lanes(256, gs, chunks)
        chain += ceil(chunks, lanes) + TREE * ceil(chunks, 8 * lanes)
    return chain


def longest(spec, shape, dtype, backward):
    return max(group_norm_chain(c, shape, dtype, backward) for c in B.Plan(B.Graph.from_spec(spec)).candidates())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_listed_group_norm_shapes_add_at_most_a_hundred(dtype):
    for shape in test_gpu_group_norm.SHAPES + [(2, 33, 32, 10), (1, 60000, 32, 8), (1, 5000, 4, 10), (2, 60, 4, 8), (2, 5000, 4, 10), (300, 1, 1, 1)]:
        for backward, keep in ((False, "stats"), (False, "checkpoint"), (True, "stats"), (True, "checkpoint")):
            spec = (group_norm_backward_graph if backward else group_norm_graph)(*shape, dtype=dtype, act="silu", keep=keep)
            if B.Plan(B.Graph.from_spec(spec)).info["pattern"] != "unfused":
                assert longest(spec, shape, dtype, backward) <= 100, spec.name


def test_sums_over_very_many_entries_are_longer():
    """The gradients of gain and shift, the fold of one row per batch entry: bounds for these count what it takes."""
    assert longest(group_norm_backward_graph(20000, 1, 2, 4, "bf16", "silu", "stats"), (20000, 1, 2, 4), "bf16", True) == 337
    assert longest(group_norm_graph(20000, 1, 2, 4, "bf16", "silu", "stats"), (20000, 1, 2, 4), "bf16", False) <= 100


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_listed_bias_gradients_add_at_most_a_hundred(dtype):
    for rows, blocks, block in test_gpu_checkpoint.SHAPES:
        plan = B.Plan(B.Graph.from_spec(checkpoint_backward_graph(rows, blocks, block, dtype, "gelu", True)))
        for c in plan.candidates():
            waves, unroll, row_blocks = map(int, re.search(r"W(\d+),U(\d+),RB(\d+)", c["kernel"]).groups())
            n = ceil(rows, row_blocks * waves * unroll) * unroll + waves + folded_rows(row_blocks)
            assert n <= 100, (n, c["kernel"])
