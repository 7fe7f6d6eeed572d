"""Which groups are too wide for the group normalisation kernels, as the header says.  No GPU."""
import pytest

from paper_2009_10924_amd import binding as B
from workloads import group_norm_backward_graph, group_norm_graph


@pytest.mark.parametrize("dtype,most", [("f32", 1024), ("f16", 2048), ("bf16", 2048)])
def test_widest_groups(dtype, most):
    for shape, pattern in (((2, 300, 1, most), "group_norm"), ((1, 1, 4, most), "group_norm"), ((2, 300, 1, most + 1), "unfused"), ((1, 20000, 2, most + 1), "unfused"),
                           ((8, 196, 1, 2 * most + 1), "unfused"), ((1, 5, 1, 2 * most + 1), "unfused")):
        for keep in ("stats", "checkpoint"):
            assert B.Plan(B.Graph.from_spec(group_norm_graph(*shape, dtype=dtype, act="silu", keep=keep))).info["pattern"] == pattern, shape
            backward = pattern.replace("group_norm", "group_norm_backward")
            assert B.Plan(B.Graph.from_spec(group_norm_backward_graph(*shape, dtype=dtype, act="silu", keep=keep))).info["pattern"] == backward, shape
