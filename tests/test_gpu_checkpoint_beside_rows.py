"""8-bit tensors in graphs whose other parts are row patterns: the explorer keeps the 8-bit ops out of kernels that do not know them."""
import numpy as np
import pytest

from oracle import oracle as O
from paper_2009_10924_amd import binding as B
from workloads import make_inputs
from workloads.graphs import CHECKPOINT_TINY, E4M3_MAX, GraphSpec, OpSpec, TensorSpec

from .gpu_util import note
from .test_gpu_checkpoint import EPS, SUBNORMAL, within

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def op(out, opcode, *inputs, **attr):
    return OpSpec(out, opcode, inputs, attr)


def norm_and_checkpoint(rows, cols, dtype):
    """LayerNorm that keeps its normalised values in 8 bits, a scale per row."""
    ops = [op("mu", "reduce_mean", "x", axis=1), op("c", "sub", "x", "mu"), op("c2", "square", "c"), op("v", "reduce_mean", "c2", axis=1), op("ve", "add_scalar", "v", value=1e-5),
           op("r", "rsqrt", "ve"), op("n", "mul", "c", "r"), op("ng", "mul", "n", "gamma"), op("y", "add", "ng", "beta"),
           op("a", "abs", "n"), op("m", "reduce_max", "a", axis=1), op("s0", "scale", "m", value=1.0 / E4M3_MAX), op("s", "add_scalar", "s0", value=CHECKPOINT_TINY),
           op("q_d", "div", "n", "s"), op("q", "convert", "q_d", dtype="e4m3")]
    return GraphSpec(f"pattern_norm_checkpoint_{dtype}_{rows}x{cols}", [TensorSpec("x", dtype, (rows, cols)), TensorSpec("gamma", "f32", (cols,)), TensorSpec("beta", "f32", (cols,))],
                     ops, [("y", dtype), ("q", "e4m3"), ("s", "f32"), ("r", "f32")])


def gate_from_checkpoint(rows, cols, dtype):
    """Softmax of restored values, its largest value put away in 8 bits, and a gate by the restored values' sigmoid."""
    ops = [op("z", "mul", "q", "s"), op("m", "reduce_max", "z", axis=1), op("c", "sub", "z", "m"), op("e", "exp", "c"), op("t", "reduce_sum", "e", axis=1), op("p", "div", "e", "t"),
           op("h", "reduce_max", "p", axis=1), op("g", "sigmoid", "z"), op("w", "mul", "g", "x")]
    return GraphSpec(f"pattern_gate_checkpoint_{dtype}_{rows}x{cols}", [TensorSpec("q", "e4m3", (rows, cols)), TensorSpec("s", "f32", (rows, 1)), TensorSpec("x", dtype, (rows, cols))],
                     ops, [("p", "f32"), ("h", "e4m3"), ("w", dtype)])


def runs(spec, inp):
    import torch
    graph = B.Graph.from_spec(spec)
    dev = [B.to_device(inp[t.name], t.dtype) for t in spec.inputs]
    plan, prog = B.Plan(graph), B.Program(graph)
    for what in ("plan", "program"):
        outs = B.alloc_outputs(spec)
        for t in outs:
            t.view(torch.uint8).fill_(0xFF)
        if what == "plan":
            plan.execute(dev, outs, plan.make_workspace())
        else:
            ws = prog.make_workspace()
            prog.bind([t.data_ptr() for t in dev], [t.data_ptr() for t in outs], ws.data_ptr() if ws is not None else 0, ws.numel() if ws is not None else 0,
                      torch.cuda.current_stream().cuda_stream)()
        torch.cuda.synchronize()
        note(f"  case {spec.name} {what}")
        yield what, {n: O.to_f64(B.to_host(t, d), d) for (n, d), t in zip(spec.outputs, outs)}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(64, 128), (33, 1000), (7, 77), (2, 20000)], ids=lambda s: "x".join(map(str, s)))
def test_layernorm_with_a_checkpoint(shape, dtype):
    """Bounds as for group normalisation: means off by at most 100 u (rows / 64 lanes and their tree; 20000 values: 8 x 40 + 16)."""
    spec = norm_and_checkpoint(*shape, dtype)
    inp = make_inputs(spec, seed=1)
    env = O.evaluate(spec, inp, keep_all=True)
    steps = 100 if shape[1] < 20000 else 400
    dn = steps * U * np.abs(env["x"]).mean(1, keepdims=True) * env["r"] + 1e-5 * np.abs(env["n"])
    for what, got in runs(spec, inp):
        within(got["r"], env["r"], 1e-5 * env["r"], f"{spec.name} {what} r")
        within(got["s"], env["s"], dn.max(1, keepdims=True) / 448 + 4 * U * env["s"], f"{spec.name} {what} s")
        d = np.abs(env["q_d"])
        within(got["q"], env["q_d"], np.maximum(2.0 ** -4 * d, 2.0 ** -10) + 2 * dn / env["s"] + 8 * U * d, f"{spec.name} {what} q")
        err = dn * np.abs(env["gamma"]) + 3 * U * (np.abs(env["y"]) + np.abs(env["ng"]))
        within(got["y"], env["y"], EPS[dtype] * (np.abs(env["y"]) + err) + err + SUBNORMAL[dtype], f"{spec.name} {what} y")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(64, 128), (33, 1000), (7, 77)], ids=lambda s: "x".join(map(str, s)))
def test_rows_of_restored_values(shape, dtype):
    spec = gate_from_checkpoint(*shape, dtype)
    rng = np.random.default_rng(3)
    inp = make_inputs(spec, seed=2)
    inp["q"] = rng.integers(0, 0x70, shape).astype(np.uint8) | (rng.integers(0, 2, shape) << 7).astype(np.uint8)
    inp["s"] = (rng.uniform(0.5, 1.5, (shape[0], 1)) / 64).astype(np.float32)     # |z| up to 6
    env = O.evaluate(spec, inp, keep_all=True)
    for what, got in runs(spec, inp):
        # exp of a difference rounded to u max|z| twice, sums of up to 100 additions in a row
        p = np.abs(env["p"])
        within(got["p"], env["p"], (EPS["f32"] + 2e-5) * p, f"{spec.name} {what} p")
        h = np.abs(env["h"])
        within(got["h"], env["h"], np.maximum(2.0 ** -4 * h, 2.0 ** -10) * (1 + 1e-4) + 2e-5 * h, f"{spec.name} {what} h")
        w = np.abs(env["w"])
        within(got["w"], env["w"], (EPS[dtype] + 1e-5) * w + SUBNORMAL[dtype], f"{spec.name} {what} w")
