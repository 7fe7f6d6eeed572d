"""Backward of a block border whose branch has a bias: dh, dgamma, dx = dropout(dh) and dbias, the sum of dx over all rows, in one graph."""
import numpy as np
import pytest

import workloads as W
from oracle import oracle as O
from paper_2009_10924_amd import binding as B
from tests import operator_bounds as E
from tests.gpu_util import note, run_spec
from workloads.graphs import OpSpec

pytestmark = pytest.mark.gpu


def _spec(rows, cols, dtype, p):
    spec = W.rmsnorm_residual_backward_graph(rows, cols, dtype=dtype, p=p, sequence=3)
    spec.ops.append(OpSpec("dbias", "reduce_sum", ("dx",), {"axis": 0}))
    spec.outputs.append(("dbias", "f32"))
    spec.name += "_dbias"
    return spec


@pytest.mark.parametrize("rows,cols,dtype", [(96, 512, "bf16"), (41, 1001, "f32"), (30, 264, "f16"), (1, 4096, "bf16"), (700, 67, "f16"), (33, 4104, "f32")])
def test_every_shape(rows, cols, dtype):
    p = 0.25
    spec = _spec(rows, cols, dtype, p)
    inputs = W.make_inputs(spec, 6)
    ref = O.evaluate(spec, inputs, keep_all=True)
    kept, _ = O.dropout_kept((rows, cols), inputs["state"], p, 3)
    # the sum of a row (a lane up to 64 values, then pairwise), and the operations around it
    mean_size = np.abs(ref["gn"]).mean(1, keepdims=True)
    dh_error = np.abs(ref["r"]) * (4 * E.U32 * np.abs(ref["g"]) + np.abs(ref["nh"]) * (70 * E.U32) * (mean_size + np.abs(ref["m"]))) + \
        4 * E.U32 * (np.abs(ref["cr"]) + np.abs(ref["dres"]))
    scale = 65536.0 / (65536 - round(65536 * p))
    dx_error = kept * scale * dh_error + 2 * E.U32 * np.abs(ref["dx"])
    graph, ran = B.Graph.from_spec(spec), 0
    for i in [None] + list(range(B.Plan(graph).info["n_candidates"])):
        note(f"  case {spec.name} candidate {i}")
        try:
            got, _, info, _ = run_spec(spec, inputs, "unfused") if i is None else run_spec(spec, inputs, candidate=i)
        except B.FsError as e:
            if "scratch memory" in e.text:
                continue
            raise
        what = f"{spec.name} {info['kernel']} "
        E.close(got["dh"], ref["dh"], dtype, dh_error, what + "dh")
        E.close(got["dx"], ref["dx"], dtype, dx_error, what + "dx")
        E.close(got["dgamma"], ref["dgamma"], "f32", E.sum_error(np.abs(ref["dnh"]).sum(0, keepdims=True), 64 + 4), what + "dgamma")
        E.close(got["dbias"], ref["dbias"], "f32", dx_error.sum(0, keepdims=True) + E.sum_error(np.abs(ref["dx"]).sum(0, keepdims=True), 64), what + "dbias")
        ran += 1
    assert ran >= 2


def test_one_kernel_and_a_fold():
    info = B.Plan(B.Graph.from_spec(_spec(8192, 4096, "bf16", 0.1))).info
    assert info["pattern"] == "row_generated" and info["n_kernels"] == 2, info
    assert B.Plan(B.Graph.from_spec(_spec(1, 4096, "bf16", 0.1))).info["n_kernels"] == 1
