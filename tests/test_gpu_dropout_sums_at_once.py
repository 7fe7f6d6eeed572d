"""Backward of dropout with a bias gradient where rows and column sums run as one launch: the sums' workgroups draw the generator's numbers
again, which have to be the rows'."""
import numpy as np
import pytest

import workloads as W
from oracle import oracle as O
from paper_2009_10924_amd import binding as B
from tests import operator_bounds as E
from tests.gpu_util import note, run_spec

pytestmark = pytest.mark.gpu


def _spec(rows, cols, dtype):
    return W.dropout_backward_graph(rows, cols, 0.3, dtype=dtype, act="none", dbias=True, sequence=5)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols", [(2, 64), (2, 9), (16, 256), (33, 131), (64, 256), (16, 1024), (100, 1001), (128, 768), (7, 16)])
def test_rows_and_sums_draw_the_same(rows, cols, dtype):
    spec = _spec(rows, cols, dtype)
    inputs = W.make_inputs(spec, 3)
    note(f"  case {spec.name}")
    got, raw, info, plan = run_spec(spec, inputs, repeat=2)
    assert "at_once" in plan.describe(), info
    two = run_spec(spec, inputs, candidate=info["candidate"])
    assert "at_once" not in two[3].describe()
    assert np.array_equal(raw["g"], two[1]["g"])
    dy, ref = O.to_f64(inputs["dy"], dtype), O.evaluate(spec, inputs, keep_all=True)
    kept, _ = O.dropout_kept((rows, cols), inputs["state"], 0.3, 5)
    assert np.array_equal(got["g"] != 0.0, kept & (dy != 0.0))
    E.close(got["g"], ref["g"], dtype, 2.0 * E.U32 * np.abs(ref["g"]), "g")   # the scale's rounding and the product's
    total = np.abs(ref["g"]).sum(0, keepdims=True)
    E.close(got["dbias"], ref["dbias"], "f32", 2.0 * E.U32 * total + E.sum_error(total), "dbias")


def test_captured_and_replayed():
    import torch
    spec = _spec(64, 264, "bf16")
    inputs = W.make_inputs(spec, 3)
    plan = B.Plan(B.Graph.from_spec(spec))
    assert "at_once" in plan.describe()
    ws = plan.make_workspace()
    dev = {t.name: B.to_device(inputs[t.name], t.dtype) for t in spec.inputs}
    ins, outs, eager = [dev[t.name] for t in spec.inputs], B.alloc_outputs(spec), B.alloc_outputs(spec)
    plan.execute(ins, outs, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.execute(ins, outs, ws)
    seen = []
    for step in range(4):
        dev["state"][2] += 1
        dev["dy"].mul_(0.5)
        for t in outs:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        plan.execute(ins, eager, ws)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager))
        seen.append((outs[0] != 0).cpu())
    assert not any(torch.equal(a, b) for a, b in zip(seen, seen[1:]))


def test_over_its_input():
    """A call whose dx is dy's own memory takes the two launches: the sums' workgroups would read what the rows' have written."""
    import torch
    for dtype in ("f32", "bf16"):
        spec = _spec(64, 256, dtype)
        inputs = W.make_inputs(spec, 3)
        want = run_spec(spec, inputs, candidate=B.Plan(B.Graph.from_spec(spec)).info["candidate"])[1]
        plan = B.Plan(B.Graph.from_spec(spec))
        ws = plan.make_workspace()
        dev = {t.name: B.to_device(inputs[t.name], t.dtype) for t in spec.inputs}
        outs = B.alloc_outputs(spec)
        outs[0] = dev["dy"]
        plan.execute([dev[t.name] for t in spec.inputs], outs, ws)
        torch.cuda.synchronize()
        for t, (name, dt) in zip(outs, spec.outputs):
            assert np.array_equal(B.to_host(t, dt), want[name]), (dtype, name)
