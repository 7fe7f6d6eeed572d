"""The element-wise dropout kernel over its inputs' own memory: every form and type, at row lengths whose last group of eight is whole,
short, or the only one."""
import numpy as np
import pytest

import workloads as W
from paper_2009_10924_amd import binding as B
from tests.gpu_util import note, run_spec

pytestmark = pytest.mark.gpu

COLS = (64, 67, 7, 9, 15, 654)


def _over(spec, inputs, names):
    import torch
    note(f"  case {spec.name}")
    out, dtype = spec.outputs[0]
    _, raw, info, _ = run_spec(spec, inputs)
    assert info["pattern"] == "dropout", info
    plan = B.Plan(B.Graph.from_spec(spec))
    for name in names:
        dev = {t.name: B.to_device(inputs[t.name], t.dtype) for t in spec.inputs}
        plan.execute([dev[t.name] for t in spec.inputs], [dev[name]])
        torch.cuda.synchronize()
        assert np.array_equal(B.to_host(dev[name], dtype), raw[out]), (spec.name, name)
        for t in spec.inputs:
            if t.name != name:
                assert B.to_host(dev[t.name], t.dtype).tobytes() == inputs[t.name].tobytes(), (spec.name, name, t.name)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
def test_forward(act, dtype):
    for cols in COLS:
        for residual in (False, True):
            spec = W.dropout_graph(50, cols, 0.3, dtype=dtype, act=act, bias=True, residual=residual)
            _over(spec, W.make_inputs(spec, 2), ("x", "res") if residual else ("x",))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_backward(act, dtype):
    for cols in COLS:
        for bias in (False, True):
            spec = W.dropout_backward_graph(50, cols, 0.3, dtype=dtype, act=act, bias=bias, dbias=False)
            _over(spec, W.make_inputs(spec, 2), ("dy", "x"))
