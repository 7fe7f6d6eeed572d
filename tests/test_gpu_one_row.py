"""Sums over the only row of a pattern on both sides of where one workgroup gives way to the ops one by one: by plan, explored, and captured."""
import numpy as np
import pytest

import workloads as W
from oracle import oracle as O
from paper_2009_10924_amd import binding as B
from tests import operator_bounds as E
from tests.gpu_util import note, run_spec

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [5, 4096, 65537, 1 << 18, (1 << 20) + 3])
def test_bias_gradient_of_one_row(cols, dtype):
    import torch
    spec = W.dropout_backward_graph(1, cols, 0.2, dtype=dtype, act="none", dbias=True, sequence=7)
    inputs = W.make_inputs(spec, 3)
    note(f"  case {spec.name}")
    ref = O.evaluate(spec, inputs, keep_all=True)

    def check(got, what):
        error = 2.0 * E.U32 * np.abs(ref["g"])   # the scale's rounding and the product's; the sum of one value adds none
        E.close(got["g"], ref["g"], dtype, error, what)
        E.close(got["dbias"], ref["dbias"], "f32", error, what + " dbias")

    got, _, info, plan = run_spec(spec, inputs, repeat=2)
    assert info["pattern"] == ("unfused" if cols > 100000 else "row_generated") or 50000 < cols < 100000, info
    check(got, info["kernel"])
    program = B.Program(B.Graph.from_spec(spec))
    ins, outs = [B.to_device(inputs[t.name], t.dtype) for t in spec.inputs], B.alloc_outputs(spec)
    ws = program.make_workspace()
    args = [t.data_ptr() for t in ins], [t.data_ptr() for t in outs], ws.data_ptr(), ws.numel()
    program.bind(*args, torch.cuda.current_stream().cuda_stream)()
    torch.cuda.synchronize()
    host = lambda: {n: O.to_f64(B.to_host(t, d), d) for (n, d), t in zip(spec.outputs, outs)}  # noqa: E731
    check(host(), "explored")
    graph = torch.cuda.CUDAGraph()
    plan_ws = plan.make_workspace()
    with torch.cuda.graph(graph):
        plan.execute(ins, outs, plan_ws)
    for step in range(2):
        for t in outs:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        check(host(), f"replay {step}")
