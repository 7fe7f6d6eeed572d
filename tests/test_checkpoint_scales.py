"""Scales of an 8-bit checkpoint have one value per block of it: what only multiplies it by a float32 tensor runs op by op."""
import itertools

import pytest

from paper_2009_10924_amd import binding as B
from workloads.graphs import GraphSpec, OpSpec, TensorSpec


def product(q, s, act, dbias, dy=None):
    """z = q * s, or dy * act'(z) and its sum over the first axis."""
    result = tuple(max(a, b) for a, b in zip(q, s))
    inputs, ops = [TensorSpec("q", "e4m3", q), TensorSpec("s", "f32", s)], [OpSpec("z", "mul", ("q", "s"))]
    outputs = [("z", "f32")]
    if act:
        inputs.append(TensorSpec("dy", "f32", dy or result))
        ops += [OpSpec("da", "gelu_tanh_grad", ("z",)), OpSpec("dx", "mul", ("dy", "da"))]
        outputs = [("dx", "f32")]
    if dbias:
        ops.append(OpSpec("sum", "reduce_sum", ("dx",), {"axis": 0}))
        outputs.append(("sum", "f32"))
    return GraphSpec(f"checkpoint_backward_{q}_{s}", inputs, ops, outputs)


def pattern(spec):
    return B.Plan(B.Graph.from_spec(spec)).info["pattern"]


@pytest.mark.parametrize("act,dbias", [(False, False), (True, False), (True, True)])
def test_scales_that_stretch_the_values_are_no_checkpoint(act, dbias):
    """As many scales as q has blocks, of other extents: the result is larger than q."""
    for q, s in (((1, 4, 64), (4, 1, 1)), ((4, 1, 64), (1, 4, 1)), ((1, 6, 2, 32), (12, 1, 1, 1)), ((1, 64), (1, 1)), ((2, 3, 1), (2, 3, 1))):
        for dy in (None, q):   # (a gradient of q's own extents stretches with it)
            if q[-1] > 1 and q[:-1] != s[:-1]:
                assert pattern(product(q, s, act, dbias, dy)) == "unfused", (q, s, dy)
            else:
                assert pattern(product(q, s, act, dbias, dy)) == "checkpoint_backward", (q, s, dy)


@pytest.mark.parametrize("act,dbias", [(False, False), (True, False), (True, True)])
def test_every_pair_of_extents_is_taken_only_as_blocks_and_their_scales(act, dbias):
    for q in itertools.product((1, 2, 4), repeat=3):
        for s in itertools.product((1, 2, 4), repeat=3):
            if any(a != b and a != 1 and b != 1 for a, b in zip(q, s)):
                continue
            blocks = s == q[:2] + (1,)
            for dy in {q, tuple(max(a, b) for a, b in zip(q, s))}:
                assert (pattern(product(q, s, act, dbias, dy)) == "checkpoint_backward") == blocks, (q, s, dy)
