"""8-bit checkpoints of every rank, scales that are none of a checkpoint's, and single ops that read and write 8-bit tensors."""
import numpy as np
import pytest

from oracle import oracle as O
from paper_2009_10924_amd import binding as B
from workloads import make_inputs
from workloads.graphs import CHECKPOINT_TINY, E4M3_MAX, GraphSpec, OpSpec, TensorSpec

from .gpu_util import note, run_spec
from .test_gpu_checkpoint import EPS, bounds, within

pytestmark = pytest.mark.gpu


def store(dims, bias, dtype):
    z, inputs, ops = "x", [TensorSpec("x", dtype, dims)], []
    if bias:
        inputs.append(TensorSpec("bias", dtype, bias))
        ops.append(OpSpec("z", "add", ("x", "bias")))
        z = "z"
    ops += [OpSpec("y", "gelu_tanh", (z,)), OpSpec("a", "abs", (z,)), OpSpec("m", "reduce_max", ("a",), {"axis": len(dims) - 1}),
            OpSpec("s0", "scale", ("m",), {"value": 1.0 / E4M3_MAX}), OpSpec("s", "add_scalar", ("s0",), {"value": CHECKPOINT_TINY}), OpSpec("q", "div", (z, "s"))]
    return GraphSpec(f"checkpoint_rank{len(dims)}", inputs, ops, [("y", dtype), ("q", "e4m3"), ("s", "f32")])


def use(dims, dtype, act, axes=()):
    inputs, ops, last = [TensorSpec("q", "e4m3", dims), TensorSpec("s", "f32", dims[:-1] + (1,))], [OpSpec("z", "mul", ("q", "s"))], "z"
    outputs = [("z", dtype)]
    if act:
        inputs.append(TensorSpec("dy", dtype, dims))
        ops += [OpSpec("da", "gelu_tanh_grad", ("z",)), OpSpec("dx", "mul", ("dy", "da"))]
        outputs, last = [("dx", dtype)], "dx"
    for k, axis in enumerate(axes):
        ops.append(OpSpec("dbias" if k + 1 == len(axes) else f"t{k}", "reduce_sum", (last,), {"axis": axis}))
        last = ops[-1].out
    return GraphSpec(f"checkpoint_backward_rank{len(dims)}", inputs, ops, outputs + ([("dbias", "f32")] if axes else []))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_store_of_every_rank(dtype):
    """(`div` stored as 8 bits, without a convert: the other spelling)"""
    for k, (dims, bias) in enumerate([((1,), None), ((5000,), (5000,)), ((9, 130), (130,)), ((3, 4, 50), (1, 4, 50)), ((2, 3, 5, 64), (5, 64)), ((2, 3, 5, 33), (3, 5, 33)),
                                      ((2, 3, 5, 7), None), ((2, 1, 5, 40), (2, 1, 5, 40))]):
        spec = store(dims, bias, dtype)
        inp = make_inputs(spec, seed=k)
        ref = O.evaluate(spec, inp)
        allowed = bounds(spec, inp, ref, dtype)
        assert B.Plan(B.Graph.from_spec(spec)).info["pattern"] == "checkpoint", dims
        for i in range(B.Plan(B.Graph.from_spec(spec)).info["n_candidates"]):
            note(f"  case {dims} {bias} {dtype} {i}")
            got, _, info, _ = run_spec(spec, inp, candidate=i)
            for name, _ in spec.outputs:
                within(got[name], ref[name], allowed[name], f"{dims} {info['kernel']} {name}")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_use_of_every_rank(dtype):
    for k, (dims, act, axes) in enumerate([((1,), False, ()), ((4097,), True, ()), ((1000, 33), True, (0,)), ((9, 130), False, ()), ((2, 30, 5, 12), True, (1, 0)),
                                           ((3, 5, 2, 33), True, (0, 1, 2)), ((2, 3, 5, 7), True, ())]):
        spec = use(dims, dtype, act, axes)
        inp = make_inputs(spec, seed=k)
        ref = O.evaluate(spec, inp)
        assert B.Plan(B.Graph.from_spec(spec)).info["pattern"] == "checkpoint_backward", dims
        for i in range(B.Plan(B.Graph.from_spec(spec)).info["n_candidates"]):
            note(f"  case {dims} {axes} {dtype} {i}")
            got, _, info, _ = run_spec(spec, inp, candidate=i)
            for name, _ in spec.outputs:
                if name == "dbias":
                    allowed = 1.6e-5 * np.abs(O.to_f64(inp["dy"], dtype)).sum(axes, keepdims=True)
                else:
                    allowed = bounds(spec, inp, ref, dtype)[name]
                within(got[name], ref[name], allowed, f"{dims} {info['kernel']} {name}")


@pytest.mark.parametrize("act,axes", [(False, ()), (True, ()), (True, (0,))])
def test_scales_that_stretch_the_values(act, axes):
    """q [1,4,64] with scales [4,1,1]: as many scales as blocks, but a result four times q."""
    spec = use((1, 4, 64), "f32", act, axes)
    spec = GraphSpec(spec.name, [TensorSpec("q", "e4m3", (1, 4, 64)), TensorSpec("s", "f32", (4, 1, 1))] + [TensorSpec("dy", "f32", (4, 4, 64))] * act, spec.ops, spec.outputs)
    inp = make_inputs(spec, seed=1)
    ref = O.evaluate(spec, inp)
    got, _, info, _ = run_spec(spec, inp)
    assert info["pattern"] == "unfused"
    for name, _ in spec.outputs:
        dy = np.abs(inp["dy"].astype(np.float64)) if act else 0.0
        allowed = 1.6e-5 * dy.sum(0, keepdims=True) if name == "dbias" else EPS["f32"] * np.abs(ref[name]) + 1e-5 * dy
        within(got[name], ref[name], allowed, name)


@pytest.mark.parametrize("dims", [(6, 40, 64), (5, 33, 12), (3, 70, 7), (2, 3, 1)])
def test_single_ops_on_8_bit_tensors(dims):
    """Accesses of 8, 4 and 1 elements: products with broadcast operands, maxima and sums over rows and middle axes, results stored
    in 8 bits.  Values of the format are exact in float32, so maxima and what is rounded once are the oracle's to the bit."""
    spec = GraphSpec("pattern_8bit_ops", [TensorSpec("q", "e4m3", dims), TensorSpec("b", "bf16", dims[-1:])],
                     [OpSpec("p", "mul", ("q", "b")), OpSpec("m", "reduce_max", ("q",), {"axis": 1}), OpSpec("r", "reduce_max", ("q",), {"axis": 2}), OpSpec("t", "reduce_sum", ("q",), {"axis": 1}),
                      OpSpec("w", "broadcast", ("m",), {"dims": dims}), OpSpec("h", "relu", ("q",))],
                     [("p", "f32"), ("m", "e4m3"), ("r", "f32"), ("t", "f32"), ("w", "e4m3"), ("h", "e4m3")])
    inp = make_inputs(spec, seed=5)
    inp["q"] = np.random.default_rng(5).integers(0, 255, dims).astype(np.uint8)
    inp["q"][(inp["q"] & 0x7F) == 0x7F] = 0x70
    ref = O.evaluate(spec, inp)
    got, _, info, _ = run_spec(spec, inp)
    assert info["pattern"] == "unfused"
    for name, d in spec.outputs:
        if name == "t":
            within(got[name], ref[name], 100 * 2.0 ** -24 * np.abs(O.to_f64(inp["q"], "e4m3")).sum(1, keepdims=True), name)
        elif name == "p":   # 4 bits times 8: exact
            assert np.array_equal(got[name], ref[name])
        else:
            assert np.array_equal(got[name], O.round_to(ref[name], d) if d == "e4m3" else ref[name]), name
