"""The 8-bit norm's float32 outputs beside one another: what it stores is what it computes with, to the last bit, in every form and launch shape."""
import numpy as np
import pytest

import workloads as W
from paper_2009_10924_amd import binding as B
from tests.gpu_util import note, run_spec

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
