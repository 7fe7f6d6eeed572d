"""8-bit checkpoints without a GPU: the storage dtype's rules, which graphs the family takes, what the oracle says of e4m3."""
import numpy as np
import pytest

from oracle import oracle as O
from paper_2009_10924_amd import binding as B
from workloads import checkpoint_backward_graph, checkpoint_graph, make_inputs, quantise
from workloads.graphs import GraphSpec, OpSpec, TensorSpec


def plan(spec, scheme="auto", **opts):
    return B.Plan(B.Graph.from_spec(spec), scheme, **opts)


# ---- the storage dtype -------------------------------------------------------------------------------------------------
def test_oracle_widens_all_256_patterns():
    torch = pytest.importorskip("torch")
    bits = np.arange(256, dtype=np.uint8)
    assert np.array_equal(O.to_f64(bits, "e4m3"), torch.from_numpy(bits).view(torch.float8_e4m3fn).double().numpy(), equal_nan=True)


def test_oracle_rounds_to_the_nearest_pattern_and_saturates():
    grid = O.to_f64(np.arange(127, dtype=np.uint8), "e4m3")            # 0 .. 448, ascending
    assert grid[-1] == 448.0 and np.all(np.diff(grid) > 0)
    for lo, hi, even in zip(grid[:-1], grid[1:], range(127)):
        mid = 0.5 * (lo + hi)
        for sign in (1.0, -1.0):
            got = O.round_to(sign * np.array([lo, np.nextafter(mid, 0), mid, np.nextafter(mid, 500), hi]), "e4m3")
            tie = lo if even % 2 == 0 else hi                           # the pattern whose last bit is 0
            assert np.array_equal(got, sign * np.array([lo, lo, tie, hi, hi]))
    assert np.array_equal(O.round_to(np.array([np.inf, -np.inf, 1e30, 465.0]), "e4m3"), [448.0, -448.0, 448.0, 448.0])
    assert np.isnan(O.round_to(np.array([np.nan]), "e4m3")[0])
    x = np.random.default_rng(0).standard_normal(4000) * 50
    assert np.array_equal(O.to_f64(quantise(x, "e4m3"), "e4m3"), O.round_to(x, "e4m3"))


def test_dtype_rules():
    g = B.Graph()
    q = g.input("e4m3", (4, 32))
    with pytest.raises(B.FsError, match="FS_ERR_DTYPE"):
        g.op("transpose", [q], perm=(1, 0))
    f = g.op("convert", [q], dtype="f32")
    b = g.op("convert", [f], dtype="e4m3")
    with pytest.raises(B.FsError, match="FS_ERR_DTYPE"):
        g.output(b, "i32")
    g.output(b, "e4m3")
    g.finalize()
    p = B.Plan(g)
    assert p.info["pattern"] == "unfused" and p.info["bytes_min"] == 2 * 4 * 32
    with pytest.raises(B.FsError):
        B.Plan(g, "wave")


def test_no_kernel_that_knows_nothing_of_8_bits_takes_such_a_graph():
    """Row patterns that other families, the row program or a generated kernel would run, with one 8-bit tensor each."""
    def softmax(dt_in, dt_out):
        ops = [OpSpec("m", "reduce_max", ("x",), {"axis": 1}), OpSpec("c", "sub", ("x", "m")), OpSpec("e", "exp", ("c",)),
               OpSpec("z", "reduce_sum", ("e",), {"axis": 1}), OpSpec("y", "div", ("e", "z"))]
        return GraphSpec("pattern_softmax", [TensorSpec("x", dt_in, (64, 128))], ops, [("y", dt_out)])
    for a, b in (("e4m3", "f32"), ("f32", "e4m3"), ("e4m3", "e4m3")):
        assert plan(softmax(a, b)).info["pattern"] == "unfused"
    sums = GraphSpec("pattern_sums", [TensorSpec("x", "e4m3", (64, 128)), TensorSpec("b", "f32", (128,))],
                     [OpSpec("y", "mul", ("x", "b")), OpSpec("s", "reduce_sum", ("y",), {"axis": 0})], [("y", "f32"), ("s", "f32")])
    p = plan(sums)
    assert p.info["pattern"] == "unfused" and "at_once" not in p.describe()
    with pytest.raises(B.FsError, match="FS_ERR_UNSUPPORTED_PATTERN"):
        B.Pack([p, p])


# ---- which graphs the family takes -------------------------------------------------------------------------------------
@pytest.mark.parametrize("act,bias", [("none", False), ("none", True), ("gelu", False), ("gelu", True), ("silu", True)])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_store_is_one_launch(act, bias, dtype):
    for shape in ((1, 1, 1), (3, 2, 5), (64, 4, 32), (7, 3, 100), (5, 1, 1537), (2, 1, 70001)):
        p = plan(checkpoint_graph(*shape, dtype=dtype, act=act, bias=bias))
        assert (p.info["pattern"], p.info["n_kernels"], p.info["workspace_bytes"]) == ("checkpoint", 1, 0), shape


@pytest.mark.parametrize("act,dbias", [("none", False), ("gelu", False), ("gelu", True), ("silu", False), ("silu", True)])
def test_use_is_one_launch_and_a_fold_of_many_rows(act, dbias):
    for shape in ((1, 1, 1), (3, 2, 5), (7, 3, 100), (5, 1, 1537), (5000, 4, 32)):
        p = plan(checkpoint_backward_graph(*shape, act=act, dbias=dbias))
        folds = dbias and shape[0] > 100
        assert (p.info["pattern"], p.info["n_kernels"], p.info["workspace_bytes"] > 0) == ("checkpoint_backward", 2 if folds else 1, folds), shape
        assert "at_once" not in p.describe()


def replaced(spec, out, **attr):
    ops = [OpSpec(o.out, o.opcode, o.inputs, {**o.attr, **(attr if o.out == out else {})}) for o in spec.ops]
    return GraphSpec(spec.name, spec.inputs, ops, spec.outputs)


def test_graphs_that_only_look_like_a_checkpoint_run_op_by_op():
    spec = checkpoint_graph(8, 2, 64)
    assert plan(replaced(spec, "q_s0", value=1 / 240.0)).info["pattern"] == "checkpoint"       # another largest value is another constant
    assert plan(replaced(spec, "q_s0", value=-1 / 448.0)).info["pattern"] == "unfused"         # a negative scale
    assert plan(replaced(spec, "q_s0", value=1.0)).info["pattern"] == "unfused"                # reciprocals could be subnormal
    assert plan(replaced(spec, "s", value=0.0)).info["pattern"] == "unfused"                   # a block of zeros divides by zero
    assert plan(replaced(spec, "q_m0", axis=1)).info["pattern"] == "unfused"                   # blocks along another axis
    back = checkpoint_backward_graph(8, 2, 64, act="silu")
    assert plan(back).info["pattern"] == "checkpoint_backward"
    assert plan(replaced(back, "da_c", value=2.0)).info["pattern"] == "unfused"                # not the slope of SiLU
    assert plan(replaced(back, "dbias", axis=1)).info["pattern"] == "unfused"                  # summed over blocks, not rows
    wide = GraphSpec(back.name, [TensorSpec("q", "e4m3", (8, 2, 64)), TensorSpec("s", "f32", (8, 1, 1)), back.inputs[2]], back.ops, back.outputs)
    assert plan(wide).info["pattern"] == "unfused"                                             # one scale for several blocks
    mixed = GraphSpec(spec.name, [spec.inputs[0], TensorSpec("bias", "f32", (2, 64))], spec.ops, spec.outputs)
    assert plan(mixed).info["pattern"] == "unfused"                                            # a bias of another dtype


def test_bias_may_repeat_at_any_axis():
    spec = checkpoint_graph(6, 4, 64)
    for dims, takes in (((64,), True), ((1, 64), True), ((4, 64), True), ((1, 4, 64), True), ((6, 4, 64), True), ((4, 1), False), ((6, 1, 64), False)):
        s = GraphSpec(spec.name, [spec.inputs[0], TensorSpec("bias", "bf16", dims)], spec.ops, spec.outputs)
        assert (plan(s).info["pattern"] == "checkpoint") == takes, dims


def test_descriptors_match_their_oracle_identities():
    """What is stored and read back is the value within half a step of the format, and the gradients are those of differences."""
    spec = checkpoint_graph(4, 3, 16, "f32", "gelu")
    inp = make_inputs(spec, seed=1)
    env = O.evaluate(spec, inp, keep_all=True)
    z = inp["x"].astype(np.float64) + inp["bias"].astype(np.float64)
    assert np.abs(env["q"] * env["s"] - z).max() <= (np.abs(z).max(-1, keepdims=True) * 2.0 ** -4).max()
    assert np.all(np.abs(env["q"] * env["s"] - z) <= np.maximum(2.0 ** -4 * np.abs(z), 2.0 ** -10 * env["s"]) * (1 + 1e-12))
    for act, f in (("gelu", O.op_gelu_tanh), ("silu", lambda v: v / (1 + np.exp(-v)))):
        back = checkpoint_backward_graph(4, 3, 16, "f32", act)
        inp = make_inputs(back, seed=2)
        z = O.to_f64(inp["q"], "e4m3") * inp["s"].astype(np.float64)
        h = 1e-5
        slope = (f(z + h) - f(z - h)) / (2 * h)
        ref = O.evaluate(back, inp)
        assert np.allclose(ref["dx"], inp["dy"].astype(np.float64) * slope, rtol=1e-7, atol=1e-8)
        assert np.allclose(ref["dbias"], (inp["dy"].astype(np.float64) * slope).sum(0, keepdims=True), rtol=1e-6, atol=1e-6)
