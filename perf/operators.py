"""Group normalisation with an activation (channels last), activation checkpoints in 8 bits, and their backward passes.

Where `own` is true, `run` makes the calls of a program built on this library: the subgraph was described and planned
once, its buffers were bound, and a pass is the bound call.  Otherwise it computes the same in plain torch.

  listed()             the cases
  draw(rng)            one more case of the same ranges
  prepare(case, seed)  inputs (made from the seed alone); plan and bound call where `own` is true
  run(state)           one pass; returns the outputs
  work(case)           bytes and operations that a pass cannot do without
  exact(case, seed)    what `run` returns, from the definition, in float64
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda"
DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
E4M3_MAX = 448.0
TINY = 1e-30   # added to a block's scale: a block of zeros divides by it
EPS = 1e-5


def listed():
    return [
        # one short sequence at inference, nothing kept for a backward pass: the latency of a call
        {"name": "group_norm_small", "kind": "group_norm", "batch": 1, "positions": 64, "groups": 32, "dim": 8, "act": "none", "keep": "none",
         "dtype": "f16"},
        # a training step's layer of 320 channels over 64 x 64 positions, groups of 10 channels, the normalised input kept in 8 bits
        {"name": "group_norm_checkpoint", "kind": "group_norm", "batch": 8, "positions": 4096, "groups": 32, "dim": 10, "act": "silu",
         "keep": "checkpoint", "dtype": "bf16"},
        # the first layers at high resolution: few channels, very many positions, statistics kept
        {"name": "group_norm_large", "kind": "group_norm", "batch": 16, "positions": 16384, "groups": 32, "dim": 8, "act": "silu", "keep": "stats",
         "dtype": "bf16"},
        # odd numbers of positions and channels, float32
        {"name": "group_norm_backward_ragged", "kind": "group_norm_backward", "batch": 3, "positions": 197, "groups": 5, "dim": 7, "act": "none",
         "keep": "stats", "dtype": "f32"},
        # the backward pass of group_norm_checkpoint
        {"name": "group_norm_backward_checkpoint", "kind": "group_norm_backward", "batch": 8, "positions": 4096, "groups": 32, "dim": 10,
         "act": "silu", "keep": "checkpoint", "dtype": "bf16"},
        # a large layer's backward pass from its input and statistics
        {"name": "group_norm_backward_large", "kind": "group_norm_backward", "batch": 8, "positions": 16384, "groups": 32, "dim": 16, "act": "gelu",
         "keep": "stats", "dtype": "f16"},
        # a small activation put away as it is
        {"name": "checkpoint_small", "kind": "checkpoint", "rows": 64, "blocks": 4, "block": 32, "act": "none", "bias": False, "dtype": "f32"},
        # bias + GELU of a feed-forward layer that keeps its pre-activation in 8 bits, a scale per 128 values
        {"name": "checkpoint_gelu", "kind": "checkpoint", "rows": 16384, "blocks": 32, "block": 128, "act": "gelu", "bias": True, "dtype": "bf16"},
        # an odd number of tokens, one scale per token, a width that is no multiple of a wavefront's span
        {"name": "checkpoint_rows", "kind": "checkpoint", "rows": 4097, "blocks": 1, "block": 1000, "act": "silu", "bias": True, "dtype": "f16"},
        # a kept activation restored for the weight gradient's matrix product
        {"name": "restore", "kind": "checkpoint_backward", "rows": 8192, "blocks": 64, "block": 128, "act": "none", "dbias": False, "dtype": "bf16"},
        # the backward pass of checkpoint_gelu with the bias gradient
        {"name": "checkpoint_backward_gelu", "kind": "checkpoint_backward", "rows": 16384, "blocks": 32, "block": 128, "act": "gelu", "dbias": True,
         "dtype": "bf16"},
        # odd numbers of tokens and features in float32
        {"name": "checkpoint_backward_ragged", "kind": "checkpoint_backward", "rows": 2047, "blocks": 1, "block": 1537, "act": "silu", "dbias": True,
         "dtype": "f32"},
    ]


# ---- more cases of the same ranges -----------------------------------------------------------------------------------
MOST = 1 << 26   # elements


def _log(rng, lo, hi):
    """An integer of [lo, hi], uniform over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))))


def draw(rng):
    kind = rng.choice(("group_norm", "group_norm_backward", "checkpoint", "checkpoint_backward"))
    dtype = rng.choice(("f32", "f16", "bf16"))
    if kind.startswith("group_norm"):
        groups, dim = rng.choice((1, 4, 8, 16, 32, 32, 32)), _log(rng, 1, 64)
        positions = _log(rng, 1, 16384)
        batch = _log(rng, 1, max(1, min(32, MOST // (groups * dim * positions))))
        keep = rng.choice(("stats", "checkpoint", "none")[:3 if kind == "group_norm" else 2])
        return {"kind": kind, "batch": batch, "positions": positions, "groups": groups, "dim": dim, "act": rng.choice(("none", "silu", "silu", "gelu")),
                "keep": keep, "dtype": dtype}
    if rng.random() < 0.5:   # a scale per block of a power of two
        block = rng.choice((32, 64, 128, 128, 256))
        blocks = max(1, _log(rng, 64, 16384) // block)
    else:                    # a scale per row
        block, blocks = _log(rng, 16, 16384), 1
    rows = _log(rng, 1, max(1, min(65536, MOST // (block * blocks))))
    act = rng.choice(("none", "gelu", "gelu", "silu"))
    case = {"kind": kind, "rows": rows, "blocks": blocks, "block": block, "act": act, "dtype": dtype}
    if kind == "checkpoint":
        case["bias"] = act != "none" and rng.random() < 0.75
    else:
        case["dbias"] = act != "none" and rng.random() < 0.75
    return case


# ---- inputs ----------------------------------------------------------------------------------------------------------
def _shape(case):
    if case["kind"].startswith("group_norm"):
        return case["batch"], case["positions"], case["groups"], case["dim"]
    return case["rows"], case["blocks"], case["block"]


def _stored(z, dims):
    """z as 8-bit values and the scales of its blocks, which run along `dims`."""
    s = z.abs().amax(dims, keepdim=True) * (1.0 / E4M3_MAX) + TINY
    return (z / s).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn), s


def _inputs(case, seed):
    """Activations whose channels have means and spreads of their own, gradients ~ N(0,1), gains ~ 1 + N(0,0.1), biases and
    shifts ~ N(0,0.1); saved statistics and checkpoints are those of the activations."""
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    dtype, kind, shape = DTYPE[case["dtype"]], case["kind"], _shape(case)

    def normal(dims, mean=0.0, std=1.0):
        return torch.randn(dims, generator=g, device=DEVICE) * std + mean

    per_channel = shape[2:] if kind.startswith("group_norm") else shape[1:]
    x = (normal(shape) * normal(per_channel, 1.0, 0.2) + normal(per_channel, 0.0, 0.5)).to(dtype)
    v = {}
    if kind == "group_norm":
        v["x"] = x
    elif kind == "group_norm_backward":
        xf = x.float()
        mu = xf.mean((1, 3), keepdim=True)
        c = xf - mu
        r = torch.rsqrt((c * c).mean((1, 3), keepdim=True) + EPS)
        if case["keep"] == "checkpoint":
            v["q"], v["s"] = _stored(c * r, (1, 3))
        else:
            v["x"], v["mu"] = x, mu
        v["dy"] = normal(shape).to(dtype)
        v["r"] = r
    elif kind == "checkpoint":
        v["x"] = x
        if case["bias"]:
            v["bias"] = normal(per_channel, 0.0, 0.1).to(dtype)
    else:
        v["q"], v["s"] = _stored(x.float(), (2,))
        if case["act"] != "none":
            v["dy"] = normal(shape).to(dtype)
    if kind.startswith("group_norm"):
        v["gamma"] = normal(per_channel, 1.0, 0.1).to(dtype)
        if kind == "group_norm" or case["act"] != "none":
            v["beta"] = normal(per_channel, 0.0, 0.1).to(dtype)
    return v


# ---- the framework's calls -------------------------------------------------------------------------------------------
def _bound(case, v):
    """The subgraph planned, its outputs and workspace allocated, all of it bound."""
    import workloads as W
    from paper_2009_10924_amd import binding as B
    kind = case["kind"]
    if kind == "group_norm":
        spec = W.group_norm_graph(*_shape(case), dtype=case["dtype"], act=case["act"], keep=case["keep"], eps=EPS)
    elif kind == "group_norm_backward":
        spec = W.group_norm_backward_graph(*_shape(case), dtype=case["dtype"], act=case["act"], keep=case["keep"])
    elif kind == "checkpoint":
        spec = W.checkpoint_graph(*_shape(case), dtype=case["dtype"], act=case["act"], bias=case["bias"])
    else:
        spec = W.checkpoint_backward_graph(*_shape(case), dtype=case["dtype"], act=case["act"], dbias=case["dbias"])
    plan = B.Plan(B.Graph.from_spec(spec))
    outs, ws = B.alloc_outputs(spec), plan.make_workspace()
    tensors = [v[t.name] for t in spec.inputs]
    call = plan.bind([t.data_ptr() for t in tensors], [t.data_ptr() for t in outs], ws.data_ptr() if ws is not None else 0,
                     ws.numel() if ws is not None else 0, torch.cuda.current_stream().cuda_stream)
    return {"call": call, "outputs": outs, "keep": (plan, ws)}


def prepare(case, seed):
    state = {"case": case, "inputs": _inputs(case, seed)}
    if own:
        state["bound"] = _bound(case, state["inputs"])
    return state


def run(state):
    if own:
        state["bound"]["call"]()
        return state["bound"]["outputs"]
    return _plain(state["case"], state["inputs"])


# ---- the plain forms -------------------------------------------------------------------------------------------------
K0, K1 = math.sqrt(2.0 / math.pi), 0.044715


def _act(z, act):
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.tanh(K0 * (z + K1 * z * z * z)))
    return z


def _act_grad(z, act):
    if act == "silu":
        s = torch.sigmoid(z)
        return s * (1.0 + z * (1.0 - s))
    t = torch.tanh(K0 * (z + K1 * z * z * z))
    return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * K0 * (1.0 + 3.0 * K1 * z * z)


def _plain(case, v):
    kind, act, dtype = case["kind"], case["act"], DTYPE[case["dtype"]]
    if kind == "group_norm":
        x = v["x"].float()
        mu = x.mean((1, 3), keepdim=True)
        c = x - mu
        r = torch.rsqrt((c * c).mean((1, 3), keepdim=True) + EPS)
        n = c * r
        y = _act(n * v["gamma"].float() + v["beta"].float(), act).to(dtype)
        if case["keep"] == "checkpoint":
            return [y, *_stored(n, (1, 3)), r]
        return [y, mu, r] if case["keep"] == "stats" else [y]
    if kind == "group_norm_backward":
        n = v["q"].float() * v["s"] if case["keep"] == "checkpoint" else (v["x"].float() - v["mu"]) * v["r"]
        gamma, dz = v["gamma"].float(), v["dy"].float()
        if act != "none":
            dz = dz * _act_grad(n * gamma + v["beta"].float(), act)
        g = dz * gamma
        dx = (g - g.mean((1, 3), keepdim=True) - n * (g * n).mean((1, 3), keepdim=True)) * v["r"]
        return [dx.to(dtype), (dz * n).sum((0, 1), keepdim=True), dz.sum((0, 1), keepdim=True)]
    if kind == "checkpoint":
        z = v["x"].float()
        if case["bias"]:
            z = z + v["bias"].float()
        stored = _stored(z, (2,))
        return [_act(z, act).to(dtype), *stored] if act != "none" else [*stored]
    z = v["q"].float() * v["s"]
    if act == "none":
        return [z.to(dtype)]
    dx = v["dy"].float() * _act_grad(z, act)
    return [dx.to(dtype), dx.sum(0, keepdim=True)] if case["dbias"] else [dx.to(dtype)]


# ---- what a pass cannot do without -----------------------------------------------------------------------------------
OPS_PER_ELEMENT = {"group_norm": 8, "group_norm_backward": 16, "checkpoint": 4, "checkpoint_backward": 2}
ACT_OPS = {"none": 0, "silu": 5, "gelu": 9}


def work(case):
    """Every input read once, every output written once; operations per element."""
    kind, e, shape = case["kind"], SIZE[case["dtype"]], _shape(case)
    n = math.prod(shape)
    if kind.startswith("group_norm"):
        c, per_group = shape[2] * shape[3], 4 * shape[0] * shape[2]
        forward = kind == "group_norm"
        size = (2 * n * e + 2 * c * e) if forward else (2 * n * e + (1 if case["act"] == "none" else 2) * c * e + 8 * c)
        if case["keep"] == "checkpoint":
            size += n + 2 * per_group   # q, its scales, the reciprocal deviations
        elif case["keep"] == "stats":
            size += 2 * per_group + (0 if forward else n * e)
    else:
        size = n * e + n + 4 * shape[0] * shape[1]
        if case["act"] != "none":
            size += n * e
        if case.get("bias"):
            size += shape[1] * shape[2] * e
        if case.get("dbias"):
            size += shape[1] * shape[2] * 4
    return {"bytes": size, "flops": n * (OPS_PER_ELEMENT[kind] + ACT_OPS[case["act"]])}


# ---- the same from the definition, in float64 ------------------------------------------------------------------------
def _logistic(z):
    return 0.5 * (1.0 + torch.tanh(0.5 * z))


def _curve(z, act):
    """An activation and its derivative; GELU in its logistic form z / (1 + exp(-2 u))."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "silu":
        s, slope = _logistic(z), 1.0
    else:
        s, slope = _logistic(2.0 * K0 * z * (1.0 + K1 * z.pow(2))), 2.0 * K0 * (1.0 + 3.0 * K1 * z.pow(2))
    return z * s, s + z * s * (1.0 - s) * slope


def exact(case, seed):
    """Outputs held in fewer bits are given unrounded: the quotient an 8-bit value stands for, the value a 16-bit one does."""
    kind, act = case["kind"], case["act"]
    v = {k: t.double() for k, t in _inputs(case, seed).items()}
    if kind == "group_norm":
        b, s, g, d = _shape(case)
        flat = v["x"].permute(0, 2, 1, 3).reshape(b, g, s * d)   # a group's elements along one axis
        var, mean = torch.var_mean(flat, -1, correction=0, keepdim=True)
        r = 1.0 / torch.sqrt(var + EPS)
        normal = ((flat - mean) * r).reshape(b, g, s, d).permute(0, 2, 1, 3)
        y = _curve(normal * v["gamma"] + v["beta"], act)[0].contiguous()
        mean, r = mean.reshape(b, 1, g, 1), r.reshape(b, 1, g, 1)
        if case["keep"] == "checkpoint":
            scale = normal.abs().amax((1, 3), keepdim=True) / E4M3_MAX + TINY
            return [y, (normal / scale).contiguous(), scale, r]
        return [y, mean, r] if case["keep"] == "stats" else [y]
    if kind == "group_norm_backward":
        normal = v["q"] * v["s"] if case["keep"] == "checkpoint" else (v["x"] - v["mu"]) * v["r"]
        dz = v["dy"]
        if act != "none":
            dz = dz * _curve(normal * v["gamma"] + v["beta"], act)[1]
        per_channel = dz.sum(1, keepdim=True), (dz * normal).sum(1, keepdim=True)   # [N,1,G,D]: the group's means follow from them
        m1, m2 = ((v["gamma"] * t).sum(3, keepdim=True) / (case["positions"] * case["dim"]) for t in per_channel)
        return [v["r"] * (dz * v["gamma"] - m1 - normal * m2), per_channel[1].sum(0, keepdim=True), per_channel[0].sum(0, keepdim=True)]
    if kind == "checkpoint":
        z = v["x"] + v["bias"] if case["bias"] else v["x"]
        scale = z.abs().amax(2, keepdim=True) / E4M3_MAX + TINY
        stored = [z / scale, scale]
        return [_curve(z, act)[0], *stored] if act != "none" else stored
    z = v["q"] * v["s"]
    if act == "none":
        return [z]
    dx = v["dy"] * _curve(z, act)[1]
    return [dx, dx.sum(0, keepdim=True)] if case["dbias"] else [dx]
