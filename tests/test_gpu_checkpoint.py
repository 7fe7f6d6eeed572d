"""8-bit checkpoints on the GPU: every candidate of both families and the per-op plan against the float64 oracle.

Bounds, per element.  eps(t) is half a step of the storage type t relative to the value; float32 arithmetic is 2^-24 per
operation:
  s     z is one exact sum rounded once, then the constant's rounding, a product and a sum: 4 * 2^-24 relative
  q     against the unrounded quotient: 2^-4 of it (2^-10 below 2^-6), plus the quotient's own error of 8 * 2^-24, which can
        also move a value across a rounding border, where both neighbours are half a step away
  y     z sigma(w), |w| < 30 here: w's 4 roundings become an absolute error of the exponent, 30 * 4 * 2^-24 < 1e-5 relative
  dx    the slope is off by at most 8e-6 absolutely (1e-5 of |dy| with its product's rounding); it crosses zero
  dbias the terms' 1e-5 |dy|, and under 100 additions in a row of partial sums at 2^-24 each: 1.6e-5 of sum |dy|
"""
import numpy as np
import pytest

from oracle import oracle as O
from paper_2009_10924_amd import binding as B
from workloads import checkpoint_backward_graph, checkpoint_graph, make_inputs

from .gpu_util import note, run_spec

pytestmark = pytest.mark.gpu

EPS = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
SUBNORMAL = {"f32": 0.0, "f16": 2.0 ** -25, "bf16": 0.0}


def within(got, ref, bound, what):
    got, ref, bound = (np.asarray(a, dtype=np.float64) for a in (got, ref, bound))
    assert np.isfinite(got).all(), f"{what}: non-finite values"
    over = np.abs(got - ref) - bound
    assert over.max() <= 0, f"{what}: {np.abs(got - ref).flat[over.argmax()]:.3e} off where {np.broadcast_to(bound, ref.shape).flat[over.argmax()]:.3e} are allowed"


def bounds(spec, inp, ref, dtype):
    out = {}
    for name, _ in spec.outputs:
        r = np.abs(ref[name])
        if name == "s":
            out[name] = 4 * 2.0 ** -24 * r
        elif name == "q":
            out[name] = np.maximum(2.0 ** -4 * r, 2.0 ** -10) + 8 * 2.0 ** -24 * r
        elif name == "dbias":
            out[name] = 1.6e-5 * np.abs(O.to_f64(inp["dy"], dtype)).sum(0, keepdims=True)
        elif name == "dx":
            out[name] = EPS[dtype] * r + 1e-5 * np.abs(O.to_f64(inp["dy"], dtype)) * (1 + EPS[dtype]) + SUBNORMAL[dtype]
        else:
            out[name] = (EPS[dtype] + 1e-5) * r + SUBNORMAL[dtype]
    return out


def every_candidate(spec, inp, dtype, unfused=True, repeat=2):
    ref = O.evaluate(spec, inp)
    allowed = bounds(spec, inp, ref, dtype)
    n = B.Plan(B.Graph.from_spec(spec)).info["n_candidates"]
    for scheme, opts in ([("unfused", {})] if unfused else []) + [("auto", {"candidate": i}) for i in range(n)]:
        note(f"  case {spec.name} {scheme} {opts}")
        got, _, info, _ = run_spec(spec, inp, scheme, repeat=repeat, **opts)
        for name, _ in spec.outputs:
            within(got[name], ref[name], allowed[name], f"{spec.name}/{info['kernel']}/{name}")


# blocks of one value, shorter than one access, of a few accesses and a bit, of whole lane groups and workgroups, of more than a
# workgroup holds; one row, odd numbers of rows, many
SHAPES = [(1, 1, 1), (3, 2, 3), (5, 1, 7), (33, 4, 32), (7, 3, 100), (129, 2, 128), (65, 1, 257), (9, 1, 1000), (5, 1, 1537), (2, 3, 2049), (3, 1, 8200),
          (2, 1, 33001), (1, 2, 70000), (3000, 3, 16)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_store(shape, dtype):
    k = SHAPES.index(shape)
    for act, bias in [(("none", "gelu", "silu")[k % 3], k % 2 == 0), (("gelu", "silu", "none")[k % 3], k % 2 == 1)]:
        spec = checkpoint_graph(*shape, dtype=dtype, act=act, bias=bias)
        every_candidate(spec, make_inputs(spec, seed=k), dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_use(shape, dtype):
    k = SHAPES.index(shape)
    for act, dbias in [("none", False), (("gelu", "silu")[k % 2], True), (("silu", "gelu")[k % 2], k % 3 == 0)]:
        spec = checkpoint_backward_graph(*shape, dtype=dtype, act=act, dbias=dbias)
        every_candidate(spec, make_inputs(spec, seed=k), dtype)


def test_bias_sums_over_several_leading_axes():
    """[A, B, cols] and [A, B, blocks, block]: summed over both leading axes, a scale per block of the last one."""
    from workloads.graphs import GraphSpec, OpSpec, TensorSpec
    for dims, axes in (((5, 7, 96), (0, 1)), ((3, 5, 2, 40), (1, 0)), ((3, 5, 2, 40), (2, 1, 0)), ((3, 5, 2, 40), (0,))):
        ops = [OpSpec("z", "mul", ("q", "s")), OpSpec("da", "gelu_tanh_grad", ("z",)), OpSpec("dx", "mul", ("dy", "da"))]
        last = "dx"
        for i, a in enumerate(axes):
            ops.append(OpSpec(f"sum{i}", "reduce_sum", (last,), {"axis": a}))
            last = f"sum{i}"
        spec = GraphSpec(f"checkpoint_backward_axes_{len(dims)}", [TensorSpec("q", "e4m3", dims), TensorSpec("s", "f32", dims[:-1] + (1,)), TensorSpec("dy", "f32", dims)],
                         ops, [("dx", "f32"), (last, "f32")])
        inp = make_inputs(spec, seed=3)
        ref = O.evaluate(spec, inp)
        got, _, info, _ = run_spec(spec, inp)
        assert info["pattern"] == "checkpoint_backward"
        within(got["dx"], ref["dx"], 2.0 ** -24 * np.abs(ref["dx"]) + 1e-5 * np.abs(inp["dy"]), f"{dims} dx")
        within(got[last], ref[last], 1.6e-5 * np.abs(inp["dy"].astype(np.float64)).sum(axes, keepdims=True), f"{dims} {axes}")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_conversion_of_every_kind_of_value(dtype):
    """Per-op conversion to 8 bits and back: ties, subnormals, what saturates, NaN."""
    from workloads.graphs import GraphSpec, OpSpec, TensorSpec
    from workloads.inputs import quantise
    grid = O.to_f64(np.arange(127, dtype=np.uint8), "e4m3")
    mids = 0.5 * (grid[:-1] + grid[1:])
    x = np.concatenate([grid, mids, mids * (1 + 2.0 ** -8), mids * (1 - 2.0 ** -8), [464.0, 480.0, 1000.0, np.inf, 2.0 ** -11, 0.0]])
    x = np.concatenate([x, -x, [np.nan]])
    x = np.concatenate([x, np.zeros(-len(x) % 8)])
    for n in (len(x), len(x) - 4, len(x) - 1):   # accesses of 8, 4 and 1 elements
        stored = quantise(x[:n], dtype)
        spec = GraphSpec("pattern_convert", [TensorSpec("x", dtype, (n,))], [OpSpec("q", "convert", ("x",), {"dtype": "e4m3"}), OpSpec("y", "scale", ("q",), {"value": 2.0})],
                         [("q", "e4m3"), ("y", "f32")])
        got, raw, info, _ = run_spec(spec, {"x": stored})
        want = O.round_to(O.to_f64(stored, dtype), "e4m3")
        assert info["pattern"] == "unfused"
        assert np.array_equal(got["q"], want, equal_nan=True) and np.array_equal(got["y"], 2 * want, equal_nan=True)
        number = ~np.isnan(want)   # (the sign of a NaN says nothing)
        assert np.array_equal(np.signbit(got["q"][number]), np.signbit(want[number]))


@pytest.mark.parametrize("block", [32, 100, 1537, 33001])
def test_blocks_of_zeros_and_with_what_is_not_finite(block):
    """A block of zeros stores zeros; a NaN stays where it is and leaves its block's scale alone; an infinity makes its
    block's scale infinite, the others zero and itself NaN; the lowest values of a type are values like others."""
    rows = 6
    for dtype in ("f32", "bf16", "f16"):
        spec = checkpoint_graph(rows, 1, block, dtype=dtype, act="none", bias=False)
        low = {"f32": -3.0e38, "bf16": -3.0e38, "f16": -65504.0}[dtype]
        x = np.random.default_rng(block).standard_normal((rows, 1, block))
        x[0] = 0.0
        x[1, 0, block // 2] = np.nan
        x[2, 0, block - 1] = np.inf
        x[3, 0, 0] = low
        x[4] = 1e-39 if dtype != "f16" else 2.0 ** -24
        from workloads.inputs import quantise
        stored = quantise(x, dtype)
        exact = O.to_f64(stored, dtype)
        n = B.Plan(B.Graph.from_spec(spec)).info["n_candidates"]
        for opts in [{"candidate": i} for i in range(n)]:
            got, _, info, _ = run_spec(spec, {"x": stored}, **opts)
            what = f"{dtype} {info['kernel']}"
            q, s = got["q"], got["s"]
            assert np.array_equal(q[0], np.zeros((1, block))) and 0 < s[0, 0, 0] <= 1.1e-30, what
            assert np.isnan(q[1, 0, block // 2]) and np.isnan(q).sum() == 2, what
            keep = np.arange(block) != block // 2
            most = np.abs(exact[1, 0, keep]).max()
            within(s[1], [[most / 448.0]], 4 * 2.0 ** -24 * most / 448.0, what)
            within(q[1, 0, keep] * s[1, 0, 0], exact[1, 0, keep], np.maximum(2.0 ** -4 * np.abs(exact[1, 0, keep]), 2.0 ** -10 * s[1, 0, 0]) * (1 + 1e-5), what)
            assert np.isinf(s[2, 0, 0]) and np.isnan(q[2, 0, -1]) and np.array_equal(q[2, 0, :-1], np.zeros(block - 1)), what
            assert q[3, 0, 0] == -448.0 and abs(s[3, 0, 0] / (abs(exact[3, 0, 0]) / 448.0) - 1) < 1e-6, what
            for r in (3, 4, 5):
                within(q[r] * s[r, 0, 0], exact[r], np.maximum(2.0 ** -4 * np.abs(exact[r]), 2.0 ** -10 * s[r, 0, 0]) * (1 + 1e-5), what)
