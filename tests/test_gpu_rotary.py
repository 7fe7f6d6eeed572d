"""Rotary positions on the GPU against the float64 oracle: layouts, axes, parts of the head, far positions, folded transposes."""
import numpy as np
import pytest

import workloads as W
from oracle import oracle as O
from paper_2009_10924_amd import binding as B
from tests import operator_bounds as E
from tests.gpu_util import note, run_spec
from workloads.graphs import GraphSpec, OpSpec, TensorSpec

pytestmark = pytest.mark.gpu


def _error(a, attr, positions):
    """Cosine and sine are off by 3e-8 (the rounded eighth of a turn) and two roundings, and by the angle's own error: speed, product
    and the oracle's power are good to 8 units of 2^-53 of the angle.  Two products and a sum of the pair."""
    size = np.array(np.abs(a))
    total = sum(attr["pairs"])
    first = slice(0, 2 * total, 2) if attr.get("interleaved") else slice(0, total)
    second = slice(1, 2 * total, 2) if attr.get("interleaved") else slice(total, 2 * total)
    both = np.abs(a[..., first]) + np.abs(a[..., second])
    size[..., first] = size[..., second] = both
    size[..., 2 * total:] = 0.0
    angle = np.abs(positions.astype(np.float64)).max() if positions.size else 0.0
    return size * (5.0 * E.U32 + 8.0 * 2.0 ** -53 * angle)


def _check(spec, inputs, schemes=("unfused", "auto"), want="rotary"):
    env = O.evaluate(spec, inputs, keep_all=True)
    for scheme in schemes:
        note(f"  case {spec.name} {scheme}")
        got, _, info, _ = run_spec(spec, inputs, scheme, repeat=2)
        _compare(spec, inputs, env, got, info)
        if scheme == "auto":
            assert info["pattern"] == want and info["n_kernels"] == 1
    return info


def _compare(spec, inputs, env, got, info):
    plain = O.evaluate(spec, inputs)
    for name, dt in spec.outputs:
        op = next(o for o in spec.ops if o.opcode == "rotary" and o.inputs[0][0] == name[0])
        error, ref = _error(env[op.inputs[0]], op.attr, inputs["positions"]), env[op.out]
        if name != op.out:   # split behind the rotation
            error, ref = error.transpose(0, 2, 1, 3), ref.transpose(0, 2, 1, 3)
        assert ref.shape == plain[name].shape
        E.close(got[name], ref, dt, error, f"{spec.name} {info['kernel']} {name}")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("sections,dim", [((8,), 16), ((64,), 128), ((16, 24, 24), 128), ((14, 15), 80), ((3,), 6), ((1,), 2), ((5, 2, 1, 3), 25), ((9,), 21),
                                          ((1, 1), 64)])
def test_layouts(sections, dim, interleaved, dtype):
    for batch, seq, heads in ((1, 1, (3, 1)), (2, 13, (4, 2)), (3, 5, (5,))):
        for restart in ((False, True) if len(sections) > 1 else (False,)):
            spec = W.rotary_graph(batch, seq, heads, dim, sections, dtype=dtype, interleaved=interleaved, restart=restart)
            _check(spec, W.make_inputs(spec, 1))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("inverse", [False, True])
def test_split_heads(inverse, dtype):
    for heads, dim, sections in (((8, 2), 128, (16, 24, 24)), ((5, 5), 40, (13,)), ((1,), 16, (8,))):
        spec = W.rotary_graph(3, 37, heads, dim, sections, dtype=dtype, inverse=inverse, split=True)
        _check(spec, W.make_inputs(spec, 2))


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_every_launch_shape(dtype):
    for spec in (W.rotary_graph(2, 50, (12, 4), 128, (64,), dtype=dtype), W.rotary_graph(2, 50, (12, 4), 96, (20, 20), dtype=dtype, interleaved=True, split=True),
                 W.rotary_graph(1, 300, (1,), 64, (32,), dtype=dtype), W.rotary_graph(1, 2, (70,), 128, (64,), dtype=dtype)):
        inputs = W.make_inputs(spec, 3)
        env = O.evaluate(spec, inputs, keep_all=True)
        n = B.Plan(B.Graph.from_spec(spec)).info["n_candidates"]
        assert n >= 2
        for i in range(n):
            got, _, info, _ = run_spec(spec, inputs, candidate=i)
            note(f"  case {spec.name} {info['kernel']}")
            _compare(spec, inputs, env, got, info)


def test_far_and_negative_positions():
    spec = W.rotary_graph(1, 8, (2,), 128, (32, 32), dtype="f32", base=500000.0)
    inputs = W.make_inputs(spec, 3)
    inputs["positions"][...] = np.array([0, 1, -1, 1 << 20, (1 << 24) + 1, -(1 << 24) - 3, (1 << 31) - 1, -(1 << 31)], np.int32).reshape(1, 8, 1, 1)
    _check(spec, inputs)
    # a float32 angle would be off by a thousandth of a turn at 2^20 already; a position turned there and back returns
    back = W.rotary_graph(1, 8, (2,), 128, (32, 32), dtype="f32", base=500000.0, inverse=True)
    there = run_spec(spec, inputs)[1]["qr"]
    again = run_spec(back, {"q": there, "positions": inputs["positions"]})[0]["qr"]
    assert np.abs(again - O.to_f64(inputs["q"], "f32")).max() <= 12 * E.U32 * 2 * np.abs(there).max()


@pytest.mark.parametrize("dims,pos", [((7, 40), (7, 2)), ((40,), (2,)), ((2, 3, 9, 40), (9, 2)), ((2, 3, 9, 40), (2, 1, 9, 2)), ((2, 3, 9, 40), (2, 3, 1, 2)),
                                      ((2, 3, 9, 40), (1, 3, 1, 2)), ((2, 3, 9, 40), (2, 3, 9, 2)), ((2, 3, 9, 40), (2,)), ((1, 3, 1, 40), (1, 3, 1, 2))])
def test_positions_stretch_over_any_axes(dims, pos):
    for dtype in ("f32", "bf16"):
        spec = GraphSpec("pattern_rotary_any", [TensorSpec("q", dtype, dims), TensorSpec("positions", "i32", pos)],
                         [OpSpec("qr", "rotary", ("q", "positions"), {"base": 10000.0, "pairs": (10, 6)})], [("qr", dtype)])
        inputs = W.make_inputs(GraphSpec("pattern_x", spec.inputs[:1], [], []), 1)
        inputs["positions"] = np.random.default_rng(5).integers(-50, 4000, size=pos).astype(np.int32)
        _check(spec, inputs)


def test_wide_rows():
    """More steps in a row than a workgroup covers at once, and as many pairs as there may be."""
    for dtype, dim, pairs in (("bf16", 8200, 4096), ("f32", 5000, 1000), ("f16", 8192, 4096)):
        for interleaved in (False, True):
            spec = W.rotary_graph(1, 3, (2, 1), dim, (pairs,), dtype=dtype, interleaved=interleaved)
            _check(spec, W.make_inputs(spec, 1))


def test_values_that_are_not_numbers_stay_in_their_pair():
    spec = W.rotary_graph(1, 4, (2,), 20, (8,), dtype="f32")
    inputs = W.make_inputs(spec, 1)
    clean = run_spec(spec, inputs)[1]["qr"]
    inputs["q"][0, 1, 0, 3], inputs["q"][0, 2, 1, 17] = np.nan, np.inf
    raw = run_spec(spec, inputs)[1]["qr"]
    touched = np.zeros(raw.shape, bool)
    touched[0, 1, 0, [3, 11]] = True
    touched[0, 2, 1, 17] = True
    assert np.isnan(raw[0, 1, 0, [3, 11]]).all() and raw[0, 2, 1, 17] == np.inf
    assert np.array_equal(raw[~touched], clean[~touched])


def test_in_place_runs_op_by_op_or_is_refused():
    import torch
    spec = W.rotary_graph(2, 6, (3,), 32, (16,), dtype="f32")
    inputs = W.make_inputs(spec, 1)
    want = run_spec(spec, inputs, "unfused")[1]["qr"]
    plan = B.Plan(B.Graph.from_spec(spec))
    dev = {t.name: B.to_device(inputs[t.name], t.dtype) for t in spec.inputs}
    plan.execute([dev[t.name] for t in spec.inputs], [dev["q"]])   # the per-op plan of one op needs no workspace
    torch.cuda.synchronize()
    assert np.array_equal(B.to_host(dev["q"], "f32"), want)


def test_captured_and_replayed_with_new_positions():
    import torch
    spec = W.rotary_graph(4, 1, (8, 2), 64, (32,), dtype="bf16")
    inputs = W.make_inputs(spec, 1)
    plan = B.Plan(B.Graph.from_spec(spec))
    dev = {t.name: B.to_device(inputs[t.name], t.dtype) for t in spec.inputs}
    ins, outs, eager = [dev[t.name] for t in spec.inputs], B.alloc_outputs(spec), B.alloc_outputs(spec)
    plan.execute(ins, outs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.execute(ins, outs)
    for step in range(3):
        dev["positions"] += 1
        graph.replay()
        torch.cuda.synchronize()
        plan.execute(ins, eager)
        torch.cuda.synchronize()
        for a, b in zip(outs, eager):
            assert torch.equal(a, b)
