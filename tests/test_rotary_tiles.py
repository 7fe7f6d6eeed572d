"""A thread of the rotary kernel loads all its rows at once: no launch shape gives it more than the kernel was compiled for."""
import random
import re

from paper_2009_10924_amd import binding as B
from workloads import rotary_graph


def test_rows_of_a_thread():
    rng = random.Random(5)
    for _ in range(60):
        pairs = rng.choice((1, 3, 16, 17, 36, 64, 300))
        heads = (rng.choice((1, 2, 5, 8, 32, 127)), rng.choice((1, 2, 8)))[:rng.choice((1, 2))]
        spec = rotary_graph(rng.choice((1, 3, 16)), rng.choice((1, 7, 197, 2048)), heads, 2 * pairs + rng.choice((0, 0, 6)), (pairs,),
                            dtype=rng.choice(("f32", "bf16")), split=rng.random() < 0.5)
        for c in B.Plan(B.Graph.from_spec(spec)).candidates():
            rows, each = (int(v) for v in re.search(r",U(\d+),P\d+,H\d+x(\d+)>", c["kernel"]).groups())
            assert each <= rows and rows in (1, 2, 3, 5), (spec.name, c["kernel"])
