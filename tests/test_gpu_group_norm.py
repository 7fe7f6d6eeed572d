"""Group normalisation on the GPU: every candidate of both families and the per-op plan against the float64 oracle.

Bounds, per element, with u = 2^-24 and eps(t) half a step of the storage type t relative to the value.  No sum here is longer
than 100 additions in a row (positions in a thread, threads of a workgroup, chunks, batch), so it is off by 100 u of the sum of
its terms' sizes.
  mean   100 u mean|x|                      =: dm
  rstd   half of the variance's 100 u and of its terms' 2 u, and the instruction's 2 u: 1e-5 relative
  xh     dm rstd + 1e-5 |xh|                =: dn
  scale  its largest xh's dn / 448, and 4 u
  q      against the unrounded quotient: 2^-4 of it (2^-10 below 2^-6), dn / s, and 8 u; a border's two sides are a half step each
  y      1.13 (the largest slope) (dn |gamma| + 3 u (|z| + |xh gamma|)) + 1e-5 |y| + 2e-6 (|z| + 1) for the activation
  dz     slope's 1e-5 |dy|                  (act none: exact)
  dx     rstd (2e-5 |dy gamma| + 2e-5 mean|dy gamma| + 2e-5 |xh| mean|dy gamma xh|) + 1e-5 |dx|
  dbeta  1.6e-5 sum|dy|,  dgamma 2e-5 sum|dy xh|
"""
import numpy as np
import pytest

from oracle import oracle as O
from paper_2009_10924_amd import binding as B
from workloads import group_norm_backward_graph, group_norm_graph, make_inputs

from .gpu_util import note, run_spec
from .test_gpu_checkpoint import EPS, SUBNORMAL, within

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def forward_bounds(spec, env, act, dtype):
    x, gamma = env["x"], env["gamma"]
    mean = lambda a: np.abs(a).mean((1, 3), keepdims=True)  # noqa: E731
    dm = 100 * U * mean(x)
    r, n, z = env["r"], env["n"], env["z"]
    dn = dm * r + 1e-5 * np.abs(n)
    out = {}
    for name, _ in spec.outputs:
        if name == "mu":
            out[name] = dm
        elif name == "r":
            out[name] = 1e-5 * r
        elif name == "s":
            out[name] = dn.max((1, 3), keepdims=True) / 448 + 4 * U * env["s"]
        elif name == "q":
            d = np.abs(env["q_d"])
            out[name] = np.maximum(2.0 ** -4 * d, 2.0 ** -10) + 2 * dn / env["s"] + 8 * U * d
        else:
            y = np.abs(env[name])
            err = 1.13 * (dn * np.abs(gamma) + 3 * U * (np.abs(z) + np.abs(n * gamma)))
            if act != "none":
                err = err + 1e-5 * y + 2e-6 * (np.abs(z) + 1)
            out[name] = EPS[dtype] * (y + err) + err + SUBNORMAL[dtype]
    return out


def backward_bounds(env, dtype):
    dy, gamma, n, r = np.abs(env["dy"]), np.abs(env["gamma"]), np.abs(env["n"]), env["r"]
    mean = lambda a: a.mean((1, 3), keepdims=True)  # noqa: E731
    g = dy * gamma
    dx = r * 2e-5 * (g + mean(g) + n * mean(g * n)) + 1e-5 * np.abs(env["dx"])
    return {"dx": dx + EPS[dtype] * (np.abs(env["dx"]) + dx) + SUBNORMAL[dtype], "dbeta": 1.6e-5 * dy.sum((0, 1), keepdims=True),
            "dgamma": 2e-5 * (dy * n).sum((0, 1), keepdims=True) + 1e-30}


def every_candidate(spec, inp, allowed, env, unfused=True, repeat=2):
    ref = {name: env["q_d"] if name == "q" else env[name] for name, _ in spec.outputs}
    n = B.Plan(B.Graph.from_spec(spec)).info["n_candidates"]
    for scheme, opts in ([("unfused", {})] if unfused else []) + [("auto", {"candidate": i}) for i in range(n)]:
        note(f"  case {spec.name} {scheme} {opts}")
        got, _, info, _ = run_spec(spec, inp, scheme, repeat=repeat, **opts)
        for name, _ in spec.outputs:
            within(got[name], ref[name], allowed[name], f"{spec.name}/{info['kernel']}/{name}")


# one value, one position, groups of less than an access, of odd numbers of channels, of one channel; odd numbers of positions; one
# group of many channels; more positions than a workgroup holds
SHAPES = [(1, 1, 1, 1), (2, 1, 4, 8), (1, 64, 32, 8), (3, 197, 5, 7), (2, 33, 32, 10), (1, 1000, 2, 3), (2, 2048, 4, 16), (1, 9000, 3, 5), (5, 17, 1, 61),
          (2, 50, 8, 48), (4, 7, 16, 1), (1, 300, 1, 1500), (1, 5, 1, 2500), (33, 2, 6, 20), (1, 16384, 1, 4), (3, 2, 31, 9), (1, 3000, 32, 2)]
NAME = lambda s: "x".join(map(str, s))  # noqa: E731


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=NAME)
def test_forward(shape, dtype):
    k = SHAPES.index(shape)
    for act, keep in [(("none", "gelu", "silu")[k % 3], "checkpoint"), (("gelu", "silu", "none")[k % 3], ("stats", "none")[k % 2])]:
        spec = group_norm_graph(*shape, dtype=dtype, act=act, keep=keep)
        inp = make_inputs(spec, seed=k)
        env = O.evaluate(spec, inp, keep_all=True)
        every_candidate(spec, inp, forward_bounds(spec, env, act, dtype), env)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=NAME)
def test_backward(shape, dtype):
    k = SHAPES.index(shape)
    for act, keep in [(("gelu", "silu", "none")[k % 3], "checkpoint"), (("silu", "none", "gelu")[k % 3], "stats")]:
        spec = group_norm_backward_graph(*shape, dtype=dtype, act=act, keep=keep)
        inp = make_inputs(spec, seed=k)
        env = O.evaluate(spec, inp, keep_all=True)
        every_candidate(spec, inp, backward_bounds(env, dtype), env)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("shape", [(2, 33, 32, 10), (3, 197, 5, 7), (1, 64, 32, 8), (1, 9000, 3, 5), (4, 7, 16, 1), (2, 2048, 4, 16), (1, 60000, 32, 8)], ids=NAME)
def test_float32_parameters(shape, dtype):
    for keep in ("checkpoint", "stats"):
        spec = group_norm_graph(*shape, dtype=dtype, act="silu", keep=keep, param_dtype="f32")
        inp = make_inputs(spec, seed=5)
        env = O.evaluate(spec, inp, keep_all=True)
        every_candidate(spec, inp, forward_bounds(spec, env, "silu", dtype), env)
        spec = group_norm_backward_graph(*shape, dtype=dtype, act=("silu", "none")[keep == "stats"], keep=keep, param_dtype="f32")
        inp = make_inputs(spec, seed=5)
        env = O.evaluate(spec, inp, keep_all=True)
        every_candidate(spec, inp, backward_bounds(env, dtype), env)
