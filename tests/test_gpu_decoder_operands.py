"""Dropout, 8-bit norms and rotary positions: one tensor in two roles, 8-bit operands, a state that is positions too, calls that overlap on two
streams.  Each has to give the bits of the plain case."""
import numpy as np
import pytest

import workloads as W
from oracle import oracle as O
from paper_2009_10924_amd import binding as B
from tests.gpu_util import note, run_spec
from workloads.graphs import GraphSpec, OpSpec, TensorSpec

pytestmark = pytest.mark.gpu


def _with_one_tensor(spec, name, other):
    """`spec` with input `other` read wherever `name` was."""
    ops = [OpSpec(o.out, o.opcode, tuple(other if i == name else i for i in o.inputs), o.attr) for o in spec.ops]
    return GraphSpec(spec.name + "_one", [t for t in spec.inputs if t.name != name], ops, spec.outputs)


def _same_bits(spec, name, other, seed=3):
    inputs = W.make_inputs(spec, seed)
    inputs[name] = inputs[other].copy()
    one = _with_one_tensor(spec, name, other)
    for scheme in ("unfused", "auto"):
        note(f"  case {one.name} {scheme}")
        want, info = run_spec(spec, inputs, scheme)[1:3]
        got, now = run_spec(one, {k: v for k, v in inputs.items() if k != name}, scheme)[1:3]
        assert now["pattern"] == info["pattern"]
        for out, _ in spec.outputs:
            assert np.array_equal(got[out].view(np.uint8), want[out].view(np.uint8)), (one.name, scheme, out)


@pytest.mark.parametrize("cols", [64, 131])
def test_one_tensor_in_two_roles(cols):
    _same_bits(W.dropout_graph(21, cols, 0.3, dtype="bf16", act="silu", bias=True, residual=True), "res", "x")
    _same_bits(W.dropout_backward_graph(21, cols, 0.3, dtype="f32", act="gelu", bias=False, dbias=False), "dy", "x")
    _same_bits(W.dropout_backward_graph(21, cols, 0.3, dtype="f16", act="gelu", bias=True, dbias=True), "dy", "x")
    _same_bits(W.rmsnorm_8bit_graph(21, cols, dtype="bf16", p=0.1, bias=True), "res", "x")
    _same_bits(W.rmsnorm_8bit_graph(21, cols, dtype="f32"), "res", "x")
    _same_bits(W.rmsnorm_8bit_graph(21, cols, dtype="f32", bias=True), "gamma", "bias")


def test_queries_and_keys_of_one_tensor():
    for split in (False, True):
        _same_bits(W.rotary_graph(2, 19, (4, 4), 40, (9, 8), dtype="bf16", split=split), "k", "q")


@pytest.mark.parametrize("cols", [64, 70])
def test_operands_in_8_bits(cols):
    """Element by element what float32 operands of the same values give."""
    graphs = (W.dropout_graph(9, cols, 0.4, dtype="f32"), W.rotary_graph(3, 7, (5,), cols, (20, 11), dtype="f32"))
    for spec in graphs:
        name = spec.inputs[0].name
        narrow = GraphSpec(spec.name + "_8bit", [TensorSpec(name, "e4m3", spec.inputs[0].dims)] + spec.inputs[1:], spec.ops, spec.outputs)
        inputs = W.make_inputs(narrow, 4)
        wide = {**inputs, name: O.to_f64(inputs[name], "e4m3").astype(np.float32)}
        note(f"  case {narrow.name}")
        got, info = run_spec(narrow, inputs)[1:3]
        want = run_spec(spec, wide, "unfused")[1]
        assert info["pattern"] == "unfused"
        assert np.array_equal(got[spec.outputs[0][0]], want[spec.outputs[0][0]])


def test_a_state_that_is_positions_too():
    spec = GraphSpec("pattern_state_as_positions", [TensorSpec("x", "f32", (5, 32)), TensorSpec("state", "i32", (4,))],
                     [OpSpec("d", "dropout", ("x", "state"), {"probability": 0.5}),
                      OpSpec("y", "rotary", ("d", "state"), {"base": 100.0, "pairs": (3, 4, 2, 5)})], [("y", "f32")])
    inputs = W.make_inputs(spec, 2)
    inputs["state"] = np.array([5, 77, -3, 1 << 20], np.int32)
    ref = O.evaluate(spec, inputs)["y"]
    for scheme in ("unfused", "auto"):
        got = run_spec(spec, inputs, scheme)[0]["y"]
        # two roundings of the dropout's product, the turn's cosine, sine, products and sum (5 units); angles of 2^20 at 53 bits: 8 of them
        assert np.abs(got - ref).max() <= (8.0 * 2.0 ** -24 + 8.0 * 2.0 ** -33) * 2.0 * 2.0 * np.abs(inputs["x"]).max(), scheme


def test_calls_that_overlap_on_two_streams():
    """A plan without a workspace keeps nothing between calls: two streams may run it at once."""
    import torch
    for spec in (W.dropout_graph(2048, 1000, 0.2, dtype="f32", residual=True), W.rmsnorm_8bit_graph(2048, 1000, dtype="bf16", p=0.1, keep="stats"),
                 W.rotary_graph(4, 512, (8, 2), 64, (32,), dtype="bf16", split=True)):
        plan = B.Plan(B.Graph.from_spec(spec))
        assert plan.info["workspace_bytes"] == 0
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        ins, outs, wants = [], [], []
        for k in (0, 1):
            inputs = W.make_inputs(spec, 10 + k)
            ins.append([B.to_device(inputs[t.name], t.dtype) for t in spec.inputs])
            outs.append(B.alloc_outputs(spec))
            wants.append(run_spec(spec, inputs)[1])
        torch.cuda.synchronize()
        for _ in range(5):
            for k in (0, 1):
                plan.execute(ins[k], outs[k], stream=streams[k].cuda_stream)
        torch.cuda.synchronize()
        for k in (0, 1):
            for (name, dt), t in zip(spec.outputs, outs[k]):
                assert np.array_equal(B.to_host(t, dt).view(np.uint8), wants[k][name].view(np.uint8)), (spec.name, name, k)
