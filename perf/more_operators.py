"""What stands between the matrix products of a decoder block: dropout from a counter-based generator, the root-mean-square
norm behind a residual connection with its result in 8 bits, rotary positions of one or several axes, and their backward passes.

Where `own` is true, `run` makes the calls of a program built on this library: the subgraph was described and planned
once, its buffers were bound, and a pass is the bound call.  Otherwise it computes the same in plain torch.

  listed()             the cases
  draw(rng)            one more case of the same ranges
  prepare(case, seed)  inputs (made from the seed alone); plan and bound call where `own` is true
  run(state)           one pass; returns the outputs
  work(case)           bytes and operations that a pass cannot do without
  exact(case, seed)    what `run` returns, from the definition, in float64

Which elements a dropout keeps follows from a state of four 32-bit words (seed and offset, 64 bits each), a number that
tells apart the dropouts that share a state, and the element's place: Philox4x32-10 of the counter (row * ceil(columns / 8) +
column / 8, that number, offset) under the seed gives eight 16-bit numbers for eight neighbouring columns, the low half of a word
first; an element is kept where its number is at least round(65536 p), and scaled by 65536 / (65536 - round(65536 p)).
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEVICE = "cuda"
DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
E4M3_MAX = 448.0
TINY = 1e-30   # added to a row's scale: a row of zeros divides by it
EPS = 1e-6


def listed():
    return [
        # a short sequence's attention output joins the residual stream: the latency of a call
        {"name": "dropout_small", "kind": "dropout", "rows": 64, "cols": 128, "act": "none", "bias": False, "residual": True, "p": 0.1,
         "dtype": "f16"},
        # the end of a feed-forward layer in training: bias, dropout, residual
        {"name": "dropout_residual", "kind": "dropout", "rows": 16384, "cols": 4096, "act": "none", "bias": True, "residual": True, "p": 0.1,
         "dtype": "bf16"},
        # dropout behind a hidden layer's activation, backward, with the bias gradient
        {"name": "dropout_backward_gelu", "kind": "dropout_backward", "rows": 16384, "cols": 4096, "act": "gelu", "bias": True, "dbias": True,
         "p": 0.1, "dtype": "bf16"},
        # odd numbers of tokens and features in float32
        {"name": "dropout_backward_ragged", "kind": "dropout_backward", "rows": 2047, "cols": 1537, "act": "silu", "bias": False, "dbias": True,
         "p": 0.25, "dtype": "f32"},
        # four sequences at one token each: residual, norm and the 8-bit operand of the next product
        {"name": "norm_decode", "kind": "norm", "rows": 4, "cols": 4096, "bias": False, "residual": True, "p": 0.0, "keep": "none", "dtype": "bf16"},
        # a batch of prompts
        {"name": "norm_prompts", "kind": "norm", "rows": 8192, "cols": 4096, "bias": False, "residual": True, "p": 0.0, "keep": "none",
         "dtype": "bf16"},
        # a training step's block border: bias, dropout, residual, norm; the deviations kept; a width that is no multiple of an access
        {"name": "norm_train_ragged", "kind": "norm", "rows": 8191, "cols": 2050, "bias": True, "residual": True, "p": 0.1, "keep": "stats",
         "dtype": "f16"},
        # the backward pass of a block border: gradients of the norm's input, of the branch before its dropout, of the gains
        {"name": "norm_backward", "kind": "norm_backward", "rows": 8192, "cols": 4096, "p": 0.1, "dtype": "bf16"},
        # odd sizes in float32, no dropout
        {"name": "norm_backward_ragged", "kind": "norm_backward", "rows": 1023, "cols": 1001, "p": 0.0, "dtype": "f32"},
        # sixteen sequences at one token each, far positions
        {"name": "rotary_decode", "kind": "rotary", "batch": 16, "seq": 1, "heads": 32, "kv_heads": 8, "dim": 128, "sections": "64",
         "base": 500000.0, "interleaved": False, "restart": False, "split": False, "inverse": False, "far": 131072, "dtype": "bf16"},
        # images in a prompt: time, height and width; heads split for the attention that follows
        {"name": "rotary_axes", "kind": "rotary", "batch": 2, "seq": 8192, "heads": 32, "kv_heads": 8, "dim": 128, "sections": "16,24,24",
         "base": 1000000.0, "interleaved": False, "restart": False, "split": True, "inverse": False, "far": 16384, "dtype": "bf16"},
        # the gradient of rotated queries and keys, two axes with ladders of their own, a part of the head turned, odd extents, float32
        {"name": "rotary_backward_ragged", "kind": "rotary", "batch": 3, "seq": 197, "heads": 5, "kv_heads": 5, "dim": 80, "sections": "14,15",
         "base": 10000.0, "interleaved": True, "restart": True, "split": True, "inverse": True, "far": 4096, "dtype": "f32"},
    ]


# ---- more cases of the same ranges -----------------------------------------------------------------------------------
MOST = 1 << 26   # elements


def _log(rng, lo, hi):
    """An integer of [lo, hi], uniform over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))))


def draw(rng):
    kind = rng.choice(("dropout", "dropout_backward", "norm", "norm", "norm_backward", "rotary", "rotary"))
    dtype = rng.choice(("f32", "f16", "bf16"))
    if kind == "rotary":
        interleaved, axes = rng.random() < 0.3, rng.choice((1, 1, 2, 3))
        pairs = _log(rng, max(4, axes), 128) if rng.random() < 0.5 else rng.choice((16, 32, 40, 64, 64, 128))
        cuts = sorted(rng.sample(range(1, pairs), axes - 1))
        sections = ",".join(str(b - a) for a, b in zip([0] + cuts, cuts + [pairs]))
        dim = 2 * pairs + (rng.choice((0, 0, 0, 2 * pairs, 6)))
        kv_heads = rng.choice((1, 2, 4, 8))
        heads = kv_heads * rng.choice((1, 4, 8))
        batch = _log(rng, 1, 64)
        most = min(MOST, MOST * SIZE["bf16"] // SIZE[dtype])
        seq = _log(rng, 1, max(1, min(16384, most // (batch * (heads + kv_heads) * dim))))
        return {"kind": kind, "batch": batch, "seq": seq, "heads": heads, "kv_heads": kv_heads, "dim": dim, "sections": sections,
                "base": rng.choice((10000.0, 500000.0, 1000000.0)), "interleaved": interleaved, "restart": axes > 1 and rng.random() < 0.5,
                "split": rng.random() < 0.5, "inverse": rng.random() < 0.4, "far": rng.choice((4096, 131072, 1 << 20)), "dtype": dtype}
    cols = _log(rng, 16, 16384) if rng.random() < 0.5 else rng.choice((512, 768, 1024, 2048, 4096, 5120, 8192))
    rows = _log(rng, 1, max(1, min(65536, (MOST if kind.startswith("dropout") else MOST // 2) // cols)))
    case = {"kind": kind, "rows": rows, "cols": cols, "dtype": dtype, "p": rng.choice((0.05, 0.1, 0.1, 0.2, 0.5))}
    if kind == "dropout":
        case.update(act=rng.choice(("none", "none", "gelu", "silu")), bias=rng.random() < 0.5, residual=rng.random() < 0.5)
    elif kind == "dropout_backward":
        case.update(act=rng.choice(("none", "gelu", "silu")), bias=rng.random() < 0.5, dbias=rng.random() < 0.7)
        case["bias"] = case["bias"] and case["act"] != "none"
    elif kind == "norm":
        case.update(residual=rng.random() < 0.8, keep=rng.choice(("none", "stats")))
        if not case["residual"] or rng.random() < 0.5:
            case["p"] = 0.0
        case["bias"] = case["residual"] and rng.random() < 0.5
    elif rng.random() < 0.3:
        case["p"] = 0.0
    return case


# ---- inputs ----------------------------------------------------------------------------------------------------------
def _sections(case):
    return tuple(int(n) for n in case["sections"].split(","))


def _inputs(case, seed):
    """Activations whose channels have means and spreads of their own, gradients ~ N(0,1), gains ~ 1 + N(0,0.1), biases ~ N(0,0.1);
    kept deviations are those of the activations.  Positions count up from where a sequence stands; several axes walk over images."""
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    dtype, kind = DTYPE[case["dtype"]], case["kind"]

    def normal(dims, mean=0.0, std=1.0):
        return torch.randn(dims, generator=g, device=DEVICE) * std + mean

    def whole(low, high, dims):
        return torch.randint(low, high, dims, generator=g, device=DEVICE)

    v = {}
    if kind == "rotary":
        b, s, d, axes = case["batch"], case["seq"], case["dim"], len(_sections(case))
        for name, heads in (("q", case["heads"]), ("k", case["kv_heads"])):
            v[name] = normal((b, heads, s, d) if case["split"] and case["inverse"] else (b, s, heads, d)).to(dtype)
        start = whole(0, max(1, case["far"] - s), (b, 1))
        run = torch.arange(s, device=DEVICE)[None, :]
        if axes == 1:
            places = [start + run]
        else:   # pictures of w x w patches one after the other
            w = max(2, int(math.sqrt(s / 2)))
            places = [start + run // (w * w), start + run // w % w, start + run % w][3 - axes:]
        v["positions"] = torch.stack(places, -1).to(torch.int32)[:, :, None, :].contiguous()
        return v
    shape, cols = (case["rows"], case["cols"]), (case["cols"],)

    def activations():
        return (normal(shape) * normal(cols, 1.0, 0.2) + normal(cols, 0.0, 0.5)).to(dtype)

    if kind == "dropout":
        v["x"] = activations()
        if case["residual"]:
            v["res"] = activations()
    elif kind == "dropout_backward":
        v["dy"] = normal(shape).to(dtype)
        if case["act"] != "none":
            v["x"] = activations()
    elif kind == "norm":
        v["x"] = activations()
        if case["residual"]:
            v["res"] = activations()
        v["gamma"] = normal(cols, 1.0, 0.1).to(dtype)
    else:
        v["h"] = activations()
        v["r"] = torch.rsqrt(v["h"].float().square().mean(1, keepdim=True) + EPS)
        v["dn"], v["dres"] = normal(shape).to(dtype), normal(shape).to(dtype)
        v["gamma"] = normal(cols, 1.0, 0.1).to(dtype)
    if case.get("bias"):
        v["bias"] = normal(cols, 0.0, 0.1).to(dtype)
    if case["p"] > 0.0:
        v["state"] = whole(-(1 << 31), 1 << 31, (4,)).to(torch.int32)
    return v


# ---- the framework's calls -------------------------------------------------------------------------------------------
def _bound(case, v):
    """The subgraph planned, its outputs and workspace allocated, all of it bound."""
    import workloads as W
    from paper_2009_10924_amd import binding as B
    kind = case["kind"]
    if kind == "rotary":
        spec = W.rotary_graph(case["batch"], case["seq"], (case["heads"], case["kv_heads"]), case["dim"], _sections(case), dtype=case["dtype"],
                              base=case["base"], interleaved=case["interleaved"], restart=case["restart"], inverse=case["inverse"], split=case["split"])
    elif kind == "dropout":
        spec = W.dropout_graph(case["rows"], case["cols"], case["p"], dtype=case["dtype"], act=case["act"], bias=case["bias"], residual=case["residual"])
    elif kind == "dropout_backward":
        spec = W.dropout_backward_graph(case["rows"], case["cols"], case["p"], dtype=case["dtype"], act=case["act"], bias=case["bias"], dbias=case["dbias"])
    elif kind == "norm":
        spec = W.rmsnorm_8bit_graph(case["rows"], case["cols"], dtype=case["dtype"], bias=case["bias"], residual=case["residual"], p=case["p"],
                                    keep=case["keep"], eps=EPS)
    else:
        spec = W.rmsnorm_residual_backward_graph(case["rows"], case["cols"], dtype=case["dtype"], p=case["p"])
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
M32 = 0xFFFFFFFF


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


def _times(c, m):
    """High and low word of a 32-bit number times a constant, both held in int64."""
    low, high = m * (c & 0xFFFF), m * (c >> 16)
    return (high + (low >> 16)) >> 16, (low + ((high & 0xFFFF) << 16)) & M32


def _kept(case, v):
    """Which elements the dropout keeps."""
    rows, cols = case["rows"], case["cols"]
    groups = (cols + 7) // 8
    seed_low, seed_high, offset_low, offset_high = (v["state"][i].long() & M32 for i in range(4))
    c0 = torch.arange(rows * groups, device=DEVICE)
    c1 = torch.zeros_like(c0)
    c2, c3 = c1 + offset_low, c1 + offset_high
    for i in range(10):
        high0, low0 = _times(c0, 0xD2511F53)
        high1, low1 = _times(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = high1 ^ c1 ^ ((seed_low + i * 0x9E3779B9) & M32), low1, high0 ^ c3 ^ ((seed_high + i * 0xBB67AE85) & M32), low0
    numbers = torch.stack([half for c in (c0, c1, c2, c3) for half in (c & 0xFFFF, c >> 16)], -1)
    return numbers.view(rows, groups * 8)[:, :cols] >= round(65536 * case["p"])


def _dropped(z, case, v):
    if case["p"] == 0.0:
        return z
    return torch.where(_kept(case, v), z * (65536.0 / (65536 - round(65536 * case["p"]))), torch.zeros_like(z))


def _turned(x, positions, case):
    """The pairs of the last axis turned by their angles, which are formed in 64 bits."""
    sections = _sections(case)
    angles = []
    for a, n in enumerate(sections):
        first, of = (0, n) if case["restart"] else (sum(sections[:a]), sum(sections))
        steps = torch.arange(first, first + n, device=DEVICE, dtype=torch.float64) / of
        angles.append(positions[..., a:a + 1].double() * case["base"] ** -steps)
    angle = torch.cat(angles, -1) * (-1.0 if case["inverse"] else 1.0)
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    n = sum(sections)
    if case["interleaved"]:
        a, b = x[..., 0:2 * n:2], x[..., 1:2 * n:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = x[..., :n], x[..., n:2 * n]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((turned, x[..., 2 * n:]), -1)


def _plain(case, v):
    kind, dtype = case["kind"], DTYPE[case["dtype"]]
    if kind == "rotary":
        outs = []
        for name in ("q", "k"):
            x = v[name].float()
            if case["split"] and case["inverse"]:
                x = x.transpose(1, 2)
            y = _turned(x, v["positions"], case)
            outs.append((y.transpose(1, 2) if case["split"] and not case["inverse"] else y).to(dtype).contiguous())
        return outs
    if kind == "dropout":
        z = v["x"].float()
        if case["bias"]:
            z = z + v["bias"].float()
        y = _dropped(_act(z, case["act"]), case, v)
        return [(y + v["res"].float() if case["residual"] else y).to(dtype)]
    if kind == "dropout_backward":
        dx = _dropped(v["dy"].float(), case, v)
        if case["act"] != "none":
            z = v["x"].float()
            dx = dx * _act_grad(z + v["bias"].float() if case["bias"] else z, case["act"])
        return [dx.to(dtype), dx.sum(0, keepdim=True)] if case["dbias"] else [dx.to(dtype)]
    gamma = v["gamma"].float()
    if kind == "norm":
        h = v["x"].float()
        if case["bias"]:
            h = h + v["bias"].float()
        if case["residual"]:
            h = _dropped(h, case, v) + v["res"].float()
        r = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
        n = h * r * gamma
        s = n.abs().amax(1, keepdim=True) * (1.0 / E4M3_MAX) + TINY
        q = (n / s).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
        outs = [h.to(dtype), q, s] if case["residual"] else [q, s]
        return outs + [r] if case["keep"] == "stats" else outs
    dn = v["dn"].float()
    n = v["h"].float() * v["r"]
    g = dn * gamma
    dh = (g - n * (g * n).mean(1, keepdim=True)) * v["r"] + v["dres"].float()
    outs = [dh.to(dtype), (dn * n).sum(0, keepdim=True)]
    return outs + [_dropped(dh, case, v).to(dtype)] if case["p"] > 0.0 else outs


# ---- what a pass cannot do without -----------------------------------------------------------------------------------
ACT_OPS = {"none": 0, "silu": 5, "gelu": 9}
DRAW_OPS = 10 * 8 / 8   # rounds of two products, four xors and two additions, for eight elements


def work(case):
    """Every input read once, every output written once; operations per element."""
    kind, e = case["kind"], SIZE[case["dtype"]]
    if kind == "rotary":
        tokens, axes = case["batch"] * case["seq"], len(_sections(case))
        n = tokens * (case["heads"] + case["kv_heads"]) * case["dim"]
        return {"bytes": 2 * n * e + 4 * tokens * axes, "flops": 3 * n + 20 * tokens * sum(_sections(case))}
    rows, cols = case["rows"], case["cols"]
    n = rows * cols
    size, ops = (cols * e if case.get("bias") else 0) + (16 if case["p"] > 0.0 else 0), (DRAW_OPS + 2 if case["p"] > 0.0 else 0)
    if kind == "dropout":
        size += n * e * (3 if case["residual"] else 2)
        ops += ACT_OPS[case["act"]] + 2
    elif kind == "dropout_backward":
        size += n * e * (2 if case["act"] == "none" else 3) + (4 * cols if case["dbias"] else 0)
        ops += ACT_OPS[case["act"]] + 3
    elif kind == "norm":
        size += n * e * (3 if case["residual"] else 1) + n + cols * e + 4 * rows * (2 if case["keep"] == "stats" else 1)
        ops += 8
    else:
        size += n * e * (5 if case["p"] > 0.0 else 4) + cols * e + 4 * cols + 4 * rows
        ops += 12
    return {"bytes": size, "flops": int(n * ops)}


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


def _factors(case, state):
    """What a dropout multiplies its elements by: the generator in 64-bit integers of the host, whose products of two 32-bit
    numbers are whole."""
    rows, cols = case["rows"], case["cols"]
    if case["p"] == 0.0:
        return 1.0
    key = [int(w) & M32 for w in state.cpu().tolist()]
    u64, groups, word = np.uint64, -(-cols // 8), np.uint64(32)
    x = np.zeros((4, rows * groups), u64)
    x[0], x[2], x[3] = np.arange(rows * groups, dtype=u64), key[2], key[3]
    k0, k1 = key[0], key[1]
    for _ in range(10):
        a, b = x[0] * u64(0xD2511F53), x[2] * u64(0xCD9E8D57)
        x = np.stack(((b >> word) ^ x[1] ^ u64(k0), b & u64(M32), (a >> word) ^ x[3] ^ u64(k1), a & u64(M32)))
        k0, k1 = (k0 + 0x9E3779B9) & M32, (k1 + 0xBB67AE85) & M32
    halves = np.ascontiguousarray(x.astype("<u4").T).view("<u2").reshape(rows, groups * 8)[:, :cols]
    border = round(65536 * case["p"])
    return torch.from_numpy(np.where(halves >= border, 65536.0 / (65536 - border), 0.0)).to(DEVICE)


def exact(case, seed):
    """Outputs held in fewer bits are given unrounded: the quotient an 8-bit value stands for, the value a 16-bit one does."""
    kind, v = case["kind"], _inputs(case, seed)
    if kind == "rotary":
        sections, outs = _sections(case), []
        total = sum(sections)
        axis = [a for a, n in enumerate(sections) for _ in range(n)]
        power = [i / n for n in sections for i in range(n)] if case["restart"] else [i / total for i in range(total)]
        speed = torch.tensor([math.exp(-p * math.log(case["base"])) for p in power], dtype=torch.float64, device=DEVICE)
        angle = v["positions"].double()[..., axis] * speed
        turn = torch.polar(torch.ones_like(angle), -angle if case["inverse"] else angle)
        for name in ("q", "k"):
            x = v[name].double()
            if case["split"] and case["inverse"]:
                x = x.permute(0, 2, 1, 3)
            first = list(range(0, 2 * total, 2)) if case["interleaved"] else list(range(total))
            second = [i + (1 if case["interleaved"] else total) for i in first]
            z = torch.complex(x[..., first], x[..., second]) * turn
            y = x.clone()
            y[..., first], y[..., second] = z.real, z.imag
            outs.append((y.permute(0, 2, 1, 3) if case["split"] and not case["inverse"] else y).contiguous())
        return outs
    state = v.pop("state", None)
    v = {k: t.double() for k, t in v.items()}
    factor = _factors(case, state)
    if kind == "dropout":
        y = _curve(v["x"] + v["bias"] if case["bias"] else v["x"], case["act"])[0] * factor
        return [y + v["res"] if case["residual"] else y]
    if kind == "dropout_backward":
        dx = v["dy"] * factor
        if case["act"] != "none":
            dx = dx * _curve(v["x"] + v["bias"] if case["bias"] else v["x"], case["act"])[1]
        return [dx, dx.sum(0, keepdim=True)] if case["dbias"] else [dx]
    if kind == "norm":
        h = v["x"] + v["bias"] if case["bias"] else v["x"]
        if case["residual"]:
            h = v["res"] + h * factor
        r = 1.0 / torch.sqrt(h.pow(2).sum(1, keepdim=True) / case["cols"] + EPS)
        normal = v["gamma"] * (h * r)
        scale = torch.amax(torch.abs(normal), 1, keepdim=True) / E4M3_MAX + TINY
        outs = [h, normal / scale, scale] if case["residual"] else [normal / scale, scale]
        return outs + [r] if case["keep"] == "stats" else outs
    normal = v["h"] * v["r"]
    along = (v["dn"] * v["gamma"] * normal).sum(1, keepdim=True) / case["cols"]
    dh = v["r"] * (v["dn"] * v["gamma"] - normal * along) + v["dres"]
    outs = [dh, (v["dn"] * normal).sum(0, keepdim=True)]
    return outs + [dh * factor] if case["p"] > 0.0 else outs
