"""Group normalisation on the GPU where its other tests do not look: groups with a value that is not finite, and what is kept of them."""
import numpy as np
import pytest

from oracle import oracle as O
from paper_2009_10924_amd import binding as B
from workloads import group_norm_graph, make_inputs, quantise
from workloads.graphs import CHECKPOINT_TINY, GraphSpec

from .gpu_util import note, run_spec

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
