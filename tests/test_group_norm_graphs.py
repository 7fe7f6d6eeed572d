"""Group normalisation without a GPU: which graphs the families take, and what their descriptors compute."""
import numpy as np
import pytest

from oracle import oracle as O
from paper_2009_10924_amd import binding as B
from workloads import checkpoint_backward_graph, checkpoint_graph, checkpointed_block_graph, group_norm_backward_graph, group_norm_graph, make_inputs
from workloads.graphs import GraphSpec, OpSpec, TensorSpec


def plan(spec, scheme="auto", **opts):
    return B.Plan(B.Graph.from_spec(spec), scheme, **opts)


SHAPES = [(1, 1, 1, 1), (2, 1, 4, 8), (8, 4096, 32, 10), (16, 16384, 32, 8), (3, 197, 5, 7), (1, 16384, 1, 4), (4096, 1, 32, 16), (1, 300, 1, 1000)]


@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_every_shape_has_a_plan(act, dtype):
    for shape in SHAPES:
        for keep in ("none", "stats", "checkpoint"):
            p = plan(group_norm_graph(*shape, dtype=dtype, act=act, keep=keep))
            assert p.info["pattern"] == "group_norm" and p.info["n_kernels"] in (1, 2, 3), shape
            if keep != "none":
                p = plan(group_norm_backward_graph(*shape, dtype=dtype, act=act, keep=keep))
                assert p.info["pattern"] == "group_norm_backward" and p.info["n_kernels"] in (1, 2, 3), shape
                assert "at_once" not in p.describe()


def rewired(spec, out, inputs=None, **attr):
    ops = [OpSpec(o.out, o.opcode, (inputs or o.inputs) if o.out == out else o.inputs, {**o.attr, **(attr if o.out == out else {})}) for o in spec.ops]
    return GraphSpec(spec.name, spec.inputs, ops, spec.outputs)


def test_axes_in_either_order_and_what_is_not_group_normalisation():
    spec = group_norm_graph(2, 30, 4, 8, "f32", "silu", "checkpoint")
    swapped = rewired(rewired(spec, "mu_d", axis=1), "mu", axis=3)
    assert plan(swapped).info["pattern"] == "group_norm"
    assert plan(rewired(rewired(spec, "q_m0", axis=1), "q_m1", axis=3)).info["pattern"] == "group_norm"
    for other in (rewired(rewired(spec, "mu_d", axis=2), "mu", axis=3),        # over groups
                  rewired(spec, "c2", inputs=("x",)),                          # not about the mean
                  rewired(spec, "q_a", inputs=("c",)),                         # the scale of something else
                  rewired(spec, "y", inputs=("ng", "y_sig"))):                 # the activation of something else
        assert plan(other).info["pattern"] == "unfused"
    gamma = [spec.inputs[0], TensorSpec("gamma", "f32", (1, 8)), spec.inputs[2]]
    assert plan(GraphSpec(spec.name, gamma, spec.ops, spec.outputs)).info["pattern"] == "unfused"       # one gain for all groups
    gamma = [spec.inputs[0], TensorSpec("gamma", "f32", (1, 1, 4, 8)), spec.inputs[2]]
    assert plan(GraphSpec(spec.name, gamma, spec.ops, spec.outputs)).info["pattern"] == "group_norm"
    assert plan(GraphSpec(spec.name, spec.inputs, spec.ops, [("y", "f16")] + spec.outputs[1:])).info["pattern"] == "unfused"


def test_backward_axes_and_what_is_not_it():
    spec = group_norm_backward_graph(2, 30, 4, 8, "f32", "gelu", "stats")
    assert plan(spec).info["pattern"] == "group_norm_backward"
    assert plan(rewired(rewired(spec, "dbeta_s", axis=0), "dbeta", axis=1)).info["pattern"] == "group_norm_backward"
    for other in (rewired(spec, "dgamma_s", axis=3), rewired(spec, "gn", inputs=("dz", "n")), rewired(spec, "da", inputs=("ng",)),
                  rewired(spec, "t2", inputs=("n", "m1"))):
        try:
            assert plan(other).info["pattern"] == "unfused"
        except B.FsError as e:   # an op that nothing reads any more
            assert "neither consumed" in e.text
    swapped = GraphSpec(spec.name, spec.inputs, spec.ops, spec.outputs[::-1])
    assert plan(swapped).info["pattern"] == "group_norm_backward"
    one = group_norm_backward_graph(1, 1, 1, 1, "f32", "none", "stats")   # gain and gradient have the same extents here
    assert plan(one).info["pattern"] == "group_norm_backward"


def test_workspace_and_scratch_are_checked():
    p = plan(group_norm_graph(16, 16384, 32, 8, "bf16", "silu", "stats"))
    assert p.info["n_kernels"] in (2, 3) and p.info["workspace_bytes"] > 0
    with pytest.raises(B.FsError, match="FS_ERR_WORKSPACE"):
        p.execute_ptrs([0x1000] * 3, [0x1000] * 3, 0x1000, p.info["workspace_bytes"] - 1, 0)
    with pytest.raises(B.FsError, match="FS_ERR_ALIGN"):
        p.execute_ptrs([0x1000, 0x1008, 0x1000], [0x1000] * 3, 0x1000, p.info["workspace_bytes"], 0)


@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
def test_backward_descriptor_is_the_gradient_by_differences(act):
    """sum(dy * group_norm(x)) differentiated numerically by x, gamma and beta."""
    shape = (2, 5, 2, 3)
    fwd = group_norm_graph(*shape, dtype="f32", act=act, keep="stats")
    inp = {k: v.astype(np.float64) for k, v in make_inputs(fwd, seed=4).items()}
    dy = np.random.default_rng(5).standard_normal(shape)
    out = "z" if act == "none" else "y"

    class Exact:   # the oracle on float64 inputs
        inputs, ops, outputs = [TensorSpec(t.name, "f64", t.dims) for t in fwd.inputs], fwd.ops, fwd.outputs

    keep = O.to_f64
    O.to_f64 = lambda a, dtype: np.asarray(a, np.float64) if dtype == "f64" else keep(a, dtype)
    try:
        def loss(v):
            return float((dy * O.evaluate(Exact, v, keep_all=True)[out]).sum())
        env = O.evaluate(Exact, inp, keep_all=True)
        back = group_norm_backward_graph(*shape, dtype="f32", act=act, keep="stats")

        class ExactBack:
            inputs, ops, outputs = [TensorSpec(t.name, "f64", t.dims) for t in back.inputs], back.ops, back.outputs
        ref = O.evaluate(ExactBack, {**{k: inp[k] for k in ("x", "gamma", "beta")}, "mu": env["mu"], "r": env["r"], "dy": dy})
        h = 1e-5
        for name, grad in (("x", "dx"), ("gamma", "dgamma"), ("beta", "dbeta")):
            got = np.zeros_like(inp[name])
            for i in np.ndindex(got.shape):
                up, down = ({**inp, name: inp[name].copy()} for _ in range(2))
                up[name][i] += h
                down[name][i] -= h
                got[i] = (loss(up) - loss(down)) / (2 * h)
            assert np.allclose(ref[grad].reshape(got.shape), got, rtol=1e-6, atol=1e-7), grad
    finally:
        O.to_f64 = keep


# ---- memory the outputs may not share, and the run of all four together ------------------------------------------------------
def spaced(n, base):
    return [base + 0x10000000 * i for i in range(n)]


@pytest.mark.parametrize("spec", [group_norm_graph(2, 50, 4, 16, "bf16", "silu", "checkpoint"), group_norm_backward_graph(2, 50, 4, 16, "bf16", "gelu", "stats"),
                                  checkpoint_graph(10, 4, 32, "f16", "gelu", True), checkpoint_backward_graph(10, 4, 32, "f32", "silu", True)], ids=lambda s: s.name)
def test_outputs_that_share_memory_are_refused(spec):
    """In place, partly over an input, over another output, by the last byte: refused before anything runs."""
    p = plan(spec)
    ins, outs = spaced(len(spec.inputs), 0x100000000), spaced(len(spec.outputs), 0x200000000)
    size = int(np.prod(spec.inputs[0].dims)) * {"bf16": 2, "f16": 2, "f32": 4, "e4m3": 1}[spec.inputs[0].dtype]
    for bad in ([ins[0]] + outs[1:], [ins[0] + (size - 1) // 16 * 16] + outs[1:], outs[:-1] + [ins[-1]], outs[:-1] + [outs[0] + 16]):
        with pytest.raises(B.FsError, match="FS_ERR_INVALID_ARG.*shares memory"):
            p.execute_ptrs(ins, bad, 0x300000000, p.info["workspace_bytes"], 0)
        with pytest.raises(B.FsError, match="FS_ERR_INVALID_ARG.*shares memory"):
            p.execute_static_ptrs(ins, bad, 0)


def test_explorer_takes_the_block_apart_at_its_products():
    spec = checkpointed_block_graph(6, 64, 4, 16, 256, 64)
    prog = B.Program(B.Graph.from_spec(spec))
    text = prog.describe()
    assert prog.info["n_steps"] == prog.info["n_stages"] == 4 and prog.info["n_single_ops"] == 0
    assert [w.split("=")[1] for w in text.split() if w.startswith("pattern=")] == ["group_norm", "checkpoint", "checkpoint_backward", "group_norm_backward"]
    assert prog.info["n_joint_folds"] == 2, text      # the bias gradient's and the normalisation's, in one launch at the end
    ins, outs = spaced(len(spec.inputs), 0x100000000), spaced(len(spec.outputs), 0x400000000)
    names = [n for n, _ in spec.outputs]
    bad = list(outs)
    bad[names.index("b1_dx")] = ins[[t.name for t in spec.inputs].index("b1_dy")]
    with pytest.raises(B.FsError, match="FS_ERR_INVALID_ARG.*shares memory"):   # refused before the first of the four steps
        prog.bind(ins, bad, 0x900000000, prog.info["workspace_bytes"], 0)()


def test_few_batch_entries_need_no_fold():
    """Up to four short ones in one workgroup per set of groups: the sums are complete, nothing is folded, no workspace is needed."""
    for batch, kernels in ((1, 1), (2, 1), (3, 1), (5, 2)):
        p = plan(group_norm_backward_graph(batch, 2, 32, 4, "bf16", "silu", "checkpoint"))
        assert (p.info["n_kernels"], p.info["workspace_bytes"] > 0) == (kernels, kernels > 1), batch


def test_no_launch_asks_for_more_threads_than_32_bits_count():
    most = (1 << 31) - 1
    for spec in (group_norm_graph(most, 1, 1, 1), group_norm_graph(most // 64, 1, 64, 1, keep="stats"), group_norm_graph(1, 1, most, 1), group_norm_graph(1, most, 1, 1),
                 group_norm_backward_graph(most, 1, 1, 1), group_norm_backward_graph(1, 1, most, 1), checkpoint_graph(most, 1, 1), checkpoint_graph(1, 1, most),
                 checkpoint_backward_graph(most, 1, 1), checkpoint_backward_graph(1, most, 1), checkpoint_backward_graph(most, 1, 1, act="none")):
        p = plan(spec)
        for c in p.candidates():
            assert np.prod([int(g) * b for g, b in zip(c["grid"], c["block"])]) < 1 << 32, (spec.name, c["kernel"])
    assert plan(group_norm_graph(most, 1, 1, 1)).info["pattern"] == "unfused"     # a workgroup per value: too many
    assert plan(group_norm_backward_graph(most, 1, 1, 1)).info["pattern"] == "group_norm_backward"   # several entries per workgroup


def test_checkpoint_factors_stay_finite():
    """rstd / scale of a group of equal values is 1 / (sqrt(eps) tiny): where that is no float32, the ops run one by one."""
    for eps, tiny, pattern in ((1e-5, 1e-30, "group_norm"), (1e-12, 1e-30, "group_norm"), (1e-18, 1e-30, "unfused"), (1e-5, 1e-36, "unfused"), (0.0, 1e-30, "unfused")):
        spec = rewired(group_norm_graph(2, 9, 4, 8, "f32", "silu", "checkpoint", eps=eps), "s", value=tiny)
        assert plan(spec).info["pattern"] == pattern, (eps, tiny)
        spec = group_norm_graph(2, 9, 4, 8, "f32", "silu", "stats", eps=eps)
        assert plan(spec).info["pattern"] == "group_norm"


def test_parameters_may_be_float32_beside_16_bit_values():
    for dtype in ("f16", "bf16"):
        assert plan(group_norm_graph(2, 9, 4, 8, dtype, "silu", "checkpoint", param_dtype="f32")).info["pattern"] == "group_norm"
        for act in ("none", "gelu"):
            assert plan(group_norm_backward_graph(2, 9, 4, 8, dtype, act, "stats", param_dtype="f32")).info["pattern"] == "group_norm_backward"
    assert plan(group_norm_graph(2, 9, 4, 8, "f32", "silu", "stats", param_dtype="bf16")).info["pattern"] == "unfused"
    spec = group_norm_graph(2, 9, 4, 8, "bf16", "silu", "stats")
    mixed = GraphSpec(spec.name, [TensorSpec(t.name, "f32" if t.name == "beta" else t.dtype, t.dims) for t in spec.inputs], spec.ops, spec.outputs)
    assert plan(mixed).info["pattern"] == "unfused"
