"""The 8-bit norm's float32 outputs beside one another: what it stores is what it computes with, to the last bit, in every form and launch
shape; scales where products with the gain fall below float32's range."""
import numpy as np
import pytest

import workloads as W
from oracle import oracle as O
from paper_2009_10924_amd import binding as B
from tests import operator_bounds as E
from tests.gpu_util import note, run_spec
from tests.test_gpu_rmsnorm_8bit import _case
from workloads.graphs import RMS_EPS
from workloads.inputs import quantise

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cols", [1, 2, 3, 64, 1000, 2051, 8200, 40002])
def test_every_lane_of_a_row_has_its_deviation(cols):
    """n is h times the row's stored r, times gamma, each product rounded by itself."""
    for more in (dict(p=0.1, bias=True), {}, dict(residual=False)):
        spec = W.rmsnorm_8bit_graph(211 if cols < 8000 else 9, cols, dtype="f32", keep="stats", normed=True, **more)
        inputs = W.make_inputs(spec, 5)
        for i in range(B.Plan(B.Graph.from_spec(spec)).info["n_candidates"]):
            note(f"  case {spec.name} candidate={i}")
            _, raw, _, _ = run_spec(spec, inputs, candidate=i)
            h = raw["h"] if "h" in raw else inputs["x"]
            assert np.array_equal(raw["n"], h * raw["r"] * inputs["gamma"]), (spec.name, i)


@pytest.mark.parametrize("cols", [64, 3000, 40000])
def test_small_gains(cols):
    """h * gamma is a float32 subnormal (a few hundred of its steps, or none) where h * r * gamma is an ordinary number."""
    for gain in (1e-25, 1e-29):
        spec = W.rmsnorm_8bit_graph(3, cols, dtype="f32", residual=False, normed=True, eps=1e-37)
        rng = np.random.default_rng(7)
        inputs = {"x": (rng.uniform(0.5, 2.0, (3, cols)) * rng.choice((-1e-17, 1e-17), (3, cols))).astype(np.float32),
                  "gamma": np.full((cols,), gain, np.float32)}
        _case(3, cols, "f32", inputs=inputs, residual=False, normed=True, eps=1e-37)


@pytest.mark.parametrize("cols", [5, 64, 1000, 40000])
def test_rows_of_zeros_without_eps(cols):
    """r is infinite and n is 0 * inf: NaN, which leaves the scale alone.  Rows beside it are as they are without it."""
    spec = W.rmsnorm_8bit_graph(4, cols, dtype="f32", keep="stats", normed=True, eps=0.0)
    inputs = W.make_inputs(spec, 3)
    plain = run_spec(spec, inputs)[1]
    inputs["x"][1], inputs["res"][1] = 0.0, 0.0
    raw = run_spec(spec, inputs)[1]
    assert raw["r"][1, 0] == np.inf and np.isnan(raw["n"][1]).all() and np.isnan(O.to_f64(raw["q"], "e4m3")[1]).all()
    assert raw["s"][1, 0] == np.float32(1e-30)
    for k in (0, 2, 3):
        for name in ("h", "q", "s", "r", "n"):
            assert np.array_equal(raw[name][k], plain[name][k]), (k, name)


@pytest.mark.parametrize("cols", [1 << 20, (1 << 22) + 8, (1 << 24) - 3])
def test_very_long_rows(cols):
    """The deviation's bound is that of any row (half of what the sum of squares is off by): equal values, whose roundings all go one way,
    and positive ones."""
    rng = np.random.default_rng(11)
    for x in (np.full((1, cols), 1.7), rng.uniform(0.5, 1.5, (1, cols))):
        spec = W.rmsnorm_8bit_graph(1, cols, dtype="bf16", residual=False, keep="stats")
        inputs = W.make_inputs(spec, 3)
        inputs["x"] = quantise(x, "bf16")
        note(f"  case {spec.name}")
        got, _, info, _ = run_spec(spec, inputs)
        assert info["kernel"].startswith("rmsnorm8_long")
        h = O.to_f64(inputs["x"], "bf16")
        r = 1.0 / np.sqrt((h * h).mean(1, keepdims=True) + RMS_EPS)
        E.close(got["r"], r, "f32", r * 48.0 * E.U32, "r")
