"""Very many short groups, one per batch entry: a wavefront each does next to nothing, and past a number of them the ops one by one are
faster (their sums then run along rows).  Times beside the shapes: kernels / op by op, us, on an MI355X.  No GPU."""
import pytest

from paper_2009_10924_amd import binding as B
from workloads import group_norm_backward_graph, group_norm_graph

OP_BY_OP = [("f32", "silu", "stats", (1 << 20, 1, 1, 4)),          # 350 / 84
            ("f32", "none", "checkpoint", (1 << 22, 1, 1, 8)),     # 1622 / 506
            ("f32", "silu", "stats", (1 << 24, 1, 1, 1)),          # 4919 / 406
            ("bf16", "silu", "stats", (3360986, 1, 1, 2)),         # 1046 / 178
            ("f32", "none", "none", (272180, 2, 1, 1)),            # 83 / 38
            ("bf16", "silu", "checkpoint", (557510, 2, 1, 1)),     # 211 / 89
            ("f32", "none", "checkpoint", (903671, 1, 1, 16)),     # 346 / 216
            ("f32", "silu", "checkpoint", (925467, 2, 1, 8))]      # 378 / 275
KERNELS = [("bf16", "none", "checkpoint", (1 << 20, 1, 1, 64)),    # 522 / 845
           ("bf16", "none", "none", (1 << 15, 1, 1, 4)),           # 13 / 37
           ("f32", "silu", "stats", (919002, 2, 1, 16)),           # 311 / 348
           ("f32", "none", "checkpoint", (218228, 2, 1, 16)),      # 89 / 124
           ("bf16", "none", "none", (126575, 9, 1, 1)),            # 42 / 51
           ("bf16", "silu", "checkpoint", (6300989, 1, 2, 2)),     # 2332 / 5800
           ("f32", "silu", "none", (140930, 2, 4, 1))]             # 66 / 145


@pytest.mark.parametrize("cases,pattern", [(OP_BY_OP, "unfused"), (KERNELS, "group_norm")], ids=["op by op", "kernels"])
def test_the_faster_of_the_two(cases, pattern):
    for dtype, act, keep, shape in cases:
        assert B.Plan(B.Graph.from_spec(group_norm_graph(*shape, dtype=dtype, act=act, keep=keep))).info["pattern"] == pattern, shape
        if keep != "none":   # backward adds up over the batch, which the ops one by one are slow at
            assert B.Plan(B.Graph.from_spec(group_norm_backward_graph(*shape, dtype=dtype, act=act, keep=keep))).info["pattern"] == "group_norm_backward", shape
