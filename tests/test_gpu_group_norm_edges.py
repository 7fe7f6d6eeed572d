"""Group normalisation on the GPU where its other tests do not look: groups with a value that is not finite, and what is kept of them; a
checkpoint beside both statistics; the widest groups; sums over very many batch entries, by bounds that count their additions."""
import numpy as np
import pytest

from oracle import oracle as O
from paper_2009_10924_amd import binding as B
from workloads import group_norm_backward_graph, group_norm_graph, make_inputs, quantise
from workloads.graphs import CHECKPOINT_TINY, GraphSpec

from .gpu_util import note, run_spec
from .test_gpu_checkpoint import within
from .test_gpu_group_norm import U, backward_bounds, forward_bounds
from .test_group_norm_chains import group_norm_chain

pytestmark = pytest.mark.gpu
NAME = lambda s: "x".join(map(str, s))  # noqa: E731


def all_kept(*args, **kw):
    """y, q, s, r and mu: a checkpoint and both statistics."""
    spec = group_norm_graph(*args, keep="checkpoint", **kw)
    return GraphSpec(spec.name, spec.inputs, spec.ops, list(spec.outputs) + [("mu", "f32")])


def candidates(spec):
    return [("unfused", {})] + [("auto", {"candidate": i}) for i in range(B.Plan(B.Graph.from_spec(spec)).info["n_candidates"])]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", [(2, 60, 4, 8), (2, 5000, 4, 10), (1, 60000, 32, 8), (3, 7, 4, 3)], ids=NAME)
def test_a_group_with_a_value_that_is_not_finite(shape, dtype):
    """Its mean is none, so every one of its normalised values is NaN and kept as NaN, and neither its reciprocal deviation nor its
    scale is finite."""
    batch, positions, groups, dim = shape
    spec = all_kept(*shape, dtype=dtype, act="silu")
    inp = make_inputs(spec, seed=2)
    for poison in (np.nan, np.inf, -np.inf):
        x = O.to_f64(inp["x"], dtype).copy()
        x[batch - 1, positions // 2, 1, dim - 1] = poison
        for scheme, opts in candidates(spec):
            note(f"  case {spec.name} {poison} {scheme} {opts}")
            got, _, info, _ = run_spec(spec, {**inp, "x": quantise(x, dtype)}, scheme, **opts)
            what = (info["kernel"], poison)
            ill = {name: got[name][batch - 1, :, 1] for name, _ in spec.outputs}
            for name in ("y", "q", "r"):
                assert np.isnan(ill[name]).all(), (what, name)
            for name in ("mu", "s"):
                assert not np.isfinite(ill[name]).any(), (what, name)
            for name, _ in spec.outputs:
                got[name][batch - 1, :, 1] = 0
                assert np.isfinite(got[name]).all(), (what, name)


@pytest.mark.parametrize("shape", [(2, 60, 4, 8), (2, 5000, 4, 10), (1, 60000, 32, 8)], ids=NAME)
def test_a_group_whose_variance_is_no_float32(shape):
    """Deviations of 1e25: the variance is infinite, its root's reciprocal 0, and so are the normalised values."""
    spec = all_kept(*shape, dtype="f32", act="none")
    inp = make_inputs(spec, seed=4)
    x = inp["x"].copy()
    x[0, :, 1] *= np.float32(1e25)
    for scheme, opts in candidates(spec):
        got, _, info, _ = run_spec(spec, {**inp, "x": x}, scheme, **opts)
        assert (got["r"][0, 0, 1] == 0).all() and (got["q"][0, :, 1] == 0).all() and (got["s"][0, 0, 1] == np.float32(CHECKPOINT_TINY)).all(), info["kernel"]
        assert np.array_equal(got["z"][0, :, 1], np.broadcast_to(inp["beta"][1].astype(np.float64), got["z"][0, :, 1].shape)), info["kernel"]


def compare(spec, inp, env, allowed, pattern):
    """Every candidate of a plan that has kernels of its own; a candidate's bounds by what it launches."""
    graph = B.Graph.from_spec(spec)
    assert B.Plan(graph).info["pattern"] == pattern, spec.name
    for info in B.Plan(graph).candidates():
        note(f"  case {spec.name} {info['kernel']}")
        got, _, ran, _ = run_spec(spec, inp, candidate=info["candidate"], repeat=1)
        assert ran["kernel"] == info["kernel"] and ran["pattern"] == pattern
        bound = allowed(info)
        for name, _ in spec.outputs:
            within(got[name], env["q_d" if name == "q" else name], bound[name], f"{spec.name}/{info['kernel']}/{name}")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", [(2, 33, 32, 10), (3, 197, 5, 7), (1, 9000, 3, 5), (1, 60000, 32, 8), (4, 7, 16, 1)], ids=NAME)
def test_a_checkpoint_beside_both_statistics(shape, dtype):
    spec = all_kept(*shape, dtype=dtype, act="gelu")
    inp = make_inputs(spec, seed=8)
    env = O.evaluate(spec, inp, keep_all=True)
    allowed = forward_bounds(spec, env, "gelu", dtype)
    compare(spec, inp, env, lambda info: allowed, "group_norm")


@pytest.mark.parametrize("dtype,shape", [("f32", (1, 300, 1, 1024)), ("f32", (1, 40, 2, 999)), ("f32", (1, 5, 1, 2001)), ("f32", (3, 1, 1, 1024)),
                                         ("bf16", (1, 300, 1, 2048)), ("f16", (1, 40, 2, 1999)), ("bf16", (1, 5, 1, 3001)), ("f16", (3, 1, 1, 2048))],
                         ids=lambda v: v if isinstance(v, str) else NAME(v))
def test_the_widest_groups(dtype, shape):
    """Up to 1024 channels of a float32 group and 2048 of a 16-bit one; more where there are few positions."""
    for keep in ("checkpoint", "stats"):
        spec = group_norm_graph(*shape, dtype=dtype, act="silu", keep=keep)
        inp = make_inputs(spec, seed=9)
        env = O.evaluate(spec, inp, keep_all=True)
        allowed = forward_bounds(spec, env, "silu", dtype)
        compare(spec, inp, env, lambda info: allowed, "group_norm")
        spec = group_norm_backward_graph(*shape, dtype=dtype, act="silu", keep=keep)
        inp = make_inputs(spec, seed=9)
        env = O.evaluate(spec, inp, keep_all=True)
        allowed = backward_bounds(env, dtype)
        compare(spec, inp, env, lambda info: allowed, "group_norm_backward")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(20000, 1, 2, 4), (9000, 3, 8, 8), (3000, 2, 31, 9)], ids=NAME)
def test_sums_over_very_many_entries(shape, dtype):
    """dgamma and dbeta: 1e-5 of every term for the slope and its products (as in the other tests) and u per addition in a row, terms of
    up to 1.13 |dy| (1.13 |dy xh|) each."""
    for keep in ("checkpoint", "stats"):
        spec = group_norm_backward_graph(*shape, dtype=dtype, act="silu", keep=keep)
        inp = make_inputs(spec, seed=7)
        env = O.evaluate(spec, inp, keep_all=True)
        bound = backward_bounds(env, dtype)
        dy, n = np.abs(env["dy"]), np.abs(env["n"])

        def allowed(info):
            per_term = 1e-5 + 4 * U + 1.13 * group_norm_chain(info, shape, dtype, True) * U
            return {"dx": bound["dx"], "dbeta": per_term * dy.sum((0, 1), keepdims=True), "dgamma": per_term * (dy * n).sum((0, 1), keepdims=True)}
        compare(spec, inp, env, allowed, "group_norm_backward")


@pytest.mark.parametrize("size", [1e-19, 1e-10, 1e10, 1e18])
@pytest.mark.parametrize("shape", [(2, 60, 4, 8), (2, 5000, 4, 10), (3, 7, 4, 3)], ids=NAME)
def test_backward_of_very_small_and_very_large_values(shape, size):
    """x, its mean and its deviation times `size`, the reciprocal deviation divided by it: its square is no float32, dx still is one."""
    for act in ("none", "silu"):
        spec = group_norm_backward_graph(*shape, dtype="f32", act=act, keep="stats")
        inp = make_inputs(spec, seed=6)
        for name in ("x", "mu"):
            inp[name] = (inp[name].astype(np.float64) * size).astype(np.float32)
        inp["r"] = (inp["r"].astype(np.float64) / size).astype(np.float32)
        inp["dy"] = inp["dy"] * np.float32(8)   # (group means of g xh up to about 8)
        inp["dy"] = np.copysign(np.abs(inp["dy"]), (inp["x"] - inp["mu"]) * inp["gamma"]).astype(np.float32)
        env = O.evaluate(spec, inp, keep_all=True)
        allowed = backward_bounds(env, "f32")
        compare(spec, inp, env, lambda info: allowed, "group_norm_backward")
