"""Sums over the only row of a pattern: a row program (one workgroup) where that is faster than the ops one by one (times at the rule, in
fs_rowprog.cpp)."""
import pytest

import workloads as W
from paper_2009_10924_amd import binding as B
from workloads.graphs import GraphSpec, OpSpec, TensorSpec

pytestmark = pytest.mark.skipif(not B.codegen_available(), reason="the HIP run-time compiler is not installed here")


def _square_sum(n, rank=2):
    ops = [OpSpec("y", "square", ("x",), {}), OpSpec("s", "reduce_sum", ("y",), {"axis": 0})]
    return GraphSpec(f"square_sum_{rank}_{n}", [TensorSpec("x", "f32", (1,) * (rank - 1) + (n,))], ops, [("s", "f32")])


def _dropout(n):
    return W.dropout_backward_graph(1, n, act="gelu", bias=True, dbias=True)


@pytest.mark.parametrize("graph,cols,one_by_one", [
    (_square_sum, 2048, False), (_square_sum, 1 << 15, False), (_square_sum, 1 << 18, True), (_square_sum, 1 << 24, True), (_square_sum, 1 << 26, True),
    (_dropout, 2048, False), (_dropout, 1 << 15, False), (_dropout, 1 << 18, True), (_dropout, 1 << 24, True), (_dropout, 1 << 26, True)])
def test_no_reduction_along_the_row(graph, cols, one_by_one):
    info = B.Plan(B.Graph.from_spec(graph(cols))).info
    assert info["pattern"] == ("unfused" if one_by_one else "row_generated"), info
    assert one_by_one or info["n_kernels"] == 1


def test_any_rank():
    assert B.Plan(B.Graph.from_spec(_square_sum(4096, rank=4))).info["n_kernels"] == 1
    assert B.Plan(B.Graph.from_spec(_square_sum(1 << 22, rank=4))).info["pattern"] == "unfused"


@pytest.mark.parametrize("cols", [2048, 1 << 18, 1 << 24])
def test_a_reduction_along_the_row(cols):
    """One workgroup's either way, once instead of once for each op."""
    for spec in (W.rmsnorm_backward_graph(1, cols), W.layernorm_backward_bias_graph(1, cols), W.rmsnorm_residual_backward_graph(1, cols, p=0.1)):
        info = B.Plan(B.Graph.from_spec(spec)).info
        assert info["pattern"] == "row_generated" and info["n_kernels"] == 1, info


def test_two_rows_are_not_one():
    info = B.Plan(B.Graph.from_spec(W.dropout_backward_graph(2, 1 << 20, act="gelu", bias=True, dbias=True))).info
    assert info["pattern"] == "row_generated", info


def test_asked_for_by_scheme_or_shape():
    """What is left to choose goes op by op; what is asked for is there at any length."""
    graph = B.Graph.from_spec(_dropout(1 << 20))
    assert B.Plan(graph).info["pattern"] == "unfused"
    assert B.Plan(graph, "lds").info["pattern"] == "row_generated"
    assert B.Plan(graph, block_threads=1024).info["block"][0] == 1024
    chosen = B.Plan(graph).info
    assert chosen["candidate"] == chosen["n_candidates"] - 1 and B.Plan(graph, candidate=chosen["candidate"]).info["pattern"] == "unfused"
    assert B.Plan(graph, candidate=0).info["pattern"] == "row_generated"


@pytest.mark.parametrize("cols", [2048, 1 << 15, 1 << 17, 1 << 18, 1 << 20, 1 << 24])
@pytest.mark.parametrize("act", ["none", "gelu"])
def test_explored(act, cols):
    """The 16-bit gradient is stored rounded and summed unrounded, so its ops have to stay in one step, whichever way that runs."""
    patterns = B.Program(B.Graph.from_spec(W.dropout_backward_graph(1, cols, act=act, bias=act != "none", dbias=True))).patterns()
    info = patterns[-1]["info"]
    assert info["pattern"] == ("row_generated" if cols <= 1 << 15 else "unfused"), [p["info"]["kernel"] for p in patterns]
    assert cols > 1 << 15 or len(patterns) == 1
