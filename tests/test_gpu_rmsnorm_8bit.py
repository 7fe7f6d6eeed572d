"""The norm behind a residual connection with its result in 8 bits, on the GPU against the float64 oracle."""
import numpy as np
import pytest

import workloads as W
from oracle import oracle as O
from paper_2009_10924_amd import binding as B
from tests import operator_bounds as E
from tests.gpu_util import note, run_spec

pytestmark = pytest.mark.gpu


def _case(rows, cols, dtype, scheme="auto", inputs=None, candidate=-1, seed=1, p=0.0, bias=False, residual=True, **more):
    spec = W.rmsnorm_8bit_graph(rows, cols, dtype=dtype, p=p, bias=bias, residual=residual, **more)
    inputs = inputs or W.make_inputs(spec, seed)
    note(f"  case {spec.name} {scheme} candidate={candidate} {more}")
    got, raw, info, plan = run_spec(spec, inputs, scheme, repeat=2, **({"candidate": candidate} if candidate >= 0 else {}))
    v = {t.name: O.to_f64(inputs[t.name], t.dtype) for t in spec.inputs}
    rounded = more.get("rounded", False) and residual
    # a rounded h is what the GPU stored (ties upstream may go either way), and what follows is held to that
    ref = O.evaluate(spec, inputs, keep_all=True, stored={"h": got["h"]} if rounded and dtype != "f32" else None)
    scale = 65536.0 / (65536 - round(65536 * p))
    size = scale * (np.abs(v["x"]) + (np.abs(v["bias"]) if bias else 0.0)) + (np.abs(v["res"]) if residual else 0.0)
    h_error = 4.0 * E.U32 * size if residual else np.zeros_like(v["x"])
    if residual:
        E.close(got["h"], (O.evaluate(spec, inputs, keep_all=True)["h0"] if rounded else ref["h"]), dtype, h_error, "h")
    if rounded and dtype != "f32":
        h_error = np.zeros_like(h_error)
    h, r = ref["h" if residual else "x"], ref["r"]
    # the sum of squares (a lane adds up to 64, then lanes pairwise and wavefronts one by one), its root, and h's own error in it
    r_error = r * (48.0 * E.U32 + (np.abs(h) * h_error).mean(1, keepdims=True) * r * r)
    n_error = np.abs(ref["gamma"]) * (r * h_error + np.abs(h) * r_error) + 3.0 * E.U32 * np.abs(ref["n"])
    if more.get("keep") == "stats":
        E.close(got["r"], r, "f32", r_error, "r")
    if more.get("normed"):
        E.close(got["n"], ref["n"], dtype, n_error, "n")
    E.close(got["s"], ref["s"], "f32", n_error.max(1, keepdims=True) / 448.0 + 3.0 * E.U32 * ref["s"], "s")
    E.eight_bit(got["q"], got["s"], ref["n"], n_error, "q")
    return info


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("cols", [1, 3, 8, 9, 16, 100, 513, 1000, 2050, 4096])
def test_lengths(cols, dtype):
    for rows in (1, 2, 5, 67):
        info = _case(rows, cols, dtype, keep="stats")
        assert info["pattern"] == "rmsnorm_8bit"
    _case(3, cols, dtype, scheme="unfused", keep="stats")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_rows(dtype):
    for cols in (16384, 16387, 32768, 40001):
        info = _case(2, cols, dtype, keep="stats", normed=True, p=0.1, bias=True)
    assert info["kernel"].startswith("rmsnorm8_long")
    _case(1, 40008, dtype, residual=False, normed=True)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("cols", [136, 131])
def test_forms(cols, dtype):
    for residual, bias, p in ((False, False, 0.0), (True, False, 0.0), (True, True, 0.0), (True, False, 0.1), (True, True, 0.5)):
        for more in ({}, {"keep": "stats"}, {"normed": True}, {"rounded": True, "keep": "stats", "normed": True}):
            _case(21, cols, dtype, p=p, bias=bias, residual=residual, **more)
    if dtype != "f32":
        _case(21, cols, dtype, gain_dtype="f32", normed=True)
        _case(3, 5, dtype, gain_dtype="f32", normed=True)


@pytest.mark.parametrize("cols,dtype", [(512, "bf16"), (1000, "f16"), (2049, "f32"), (8200, "bf16"), (40, "f32")])
def test_every_launch_shape(cols, dtype):
    spec = W.rmsnorm_8bit_graph(33, cols, dtype=dtype, p=0.1, bias=True, keep="stats")
    n = B.Plan(B.Graph.from_spec(spec)).info["n_candidates"]
    assert n >= 2
    for i in range(n):
        _case(33, cols, dtype, candidate=i, p=0.1, bias=True, keep="stats")


@pytest.mark.parametrize("cols", [64, 1000, 40000])
def test_rows_of_zeros_infinities_and_nan(cols):
    """A row of zeros keeps zeros and the smallest scale; an infinity's row has r = 0, zeros and a NaN; a NaN takes its row with it.  Rows
    beside them are as they are without them."""
    spec = W.rmsnorm_8bit_graph(6, cols, dtype="f32", keep="stats", normed=True)
    inputs = W.make_inputs(spec, 3)
    plain = run_spec(spec, inputs)[1]
    bad = {k: a.copy() for k, a in inputs.items()}
    bad["x"][0], bad["res"][0] = 0.0, 0.0
    bad["x"][2, cols // 2] = np.inf
    bad["x"][4, cols - 1] = np.nan
    raw = run_spec(spec, bad)[1]
    q = O.to_f64(raw["q"], "e4m3")
    assert (q[0] == 0.0).all() and raw["s"][0, 0] == np.float32(1e-30) and (raw["n"][0] == 0.0).all()
    assert raw["r"][2, 0] == 0.0 and np.isnan(q[2, cols // 2]) and (np.delete(q[2], cols // 2) == 0.0).all() and raw["s"][2, 0] == np.float32(1e-30)
    assert np.isnan(q[4]).all() and np.isnan(raw["r"][4, 0]) and np.isnan(raw["s"][4, 0]) and np.isnan(raw["n"][4]).all()
    for k in (1, 3, 5):
        for name in ("h", "q", "s", "r", "n"):
            assert np.array_equal(raw[name][k], plain[name][k]), (k, name)


def test_gains_out_of_range():
    """h * gamma beyond float32 where h * r * gamma is not: the scale is the maximum of n."""
    for cols in (64, 3000, 40000):
        spec = W.rmsnorm_8bit_graph(3, cols, dtype="f32", residual=False, normed=True)
        inputs = W.make_inputs(spec, 3)
        inputs["x"] = (inputs["x"].astype(np.float64) * 1e15).astype(np.float32)
        inputs["gamma"] = np.full((cols,), 1e25, np.float32)
        inputs["gamma"][::2] = -3e24
        _case(3, cols, "f32", inputs=inputs, residual=False, normed=True)


def test_outputs_that_share_memory_are_refused():
    import torch
    spec = W.rmsnorm_8bit_graph(4, 64, dtype="bf16")
    inputs = W.make_inputs(spec, 3)
    plan = B.Plan(B.Graph.from_spec(spec))
    ins, outs = [B.to_device(inputs[t.name], t.dtype) for t in spec.inputs], B.alloc_outputs(spec)
    outs[0] = ins[1]
    with pytest.raises(B.FsError) as e:
        plan.execute(ins, outs)
    assert e.value.code == -1 and "shares memory" in e.value.text
    torch.cuda.synchronize()


def test_captured_and_replayed():
    import torch
    spec = W.rmsnorm_8bit_graph(70, 1000, dtype="bf16", p=0.1, bias=True, keep="stats")
    inputs = W.make_inputs(spec, 3)
    plan = B.Plan(B.Graph.from_spec(spec))
    dev = {t.name: B.to_device(inputs[t.name], t.dtype) for t in spec.inputs}
    ins, outs, eager = [dev[t.name] for t in spec.inputs], B.alloc_outputs(spec), B.alloc_outputs(spec)
    plan.execute(ins, outs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.execute(ins, outs)
    for step in range(3):
        dev["x"].mul_(0.5)
        dev["state"][3] += 1
        graph.replay()
        torch.cuda.synchronize()
        plan.execute(ins, eager)
        torch.cuda.synchronize()
        for a, b in zip(outs, eager):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
