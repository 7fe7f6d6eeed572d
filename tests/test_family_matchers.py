"""Graphs changed at random (extents, types, operands, axes, constants, outputs): whatever group normalisation and the 8-bit checkpoints
take for theirs has to mean what their kernels compute from the operands that the plan hands them.  The kernels' formulas are written
down here over flat arrays, as the kernels read them; the graph's meaning is the oracle's.  No GPU."""
import random
import re

import numpy as np
import pytest

from oracle import oracle as O
from paper_2009_10924_amd import binding as B
from workloads import checkpoint_backward_graph, checkpoint_graph, group_norm_backward_graph, group_norm_graph, quantise
from workloads.graphs import GraphSpec, OpSpec, TensorSpec

BINARY = ("add", "sub", "mul", "div", "max")
FAMILIES = ("group_norm", "group_norm_backward", "checkpoint", "checkpoint_backward")


def activated(z, act):
    return z if act == "none" else z * O.op_sigmoid(z) if act == "silu" else O.op_gelu_tanh(z)


def slope(z, act):
    if act == "silu":
        s = O.op_sigmoid(z)
        return s * (1 + z * (1 - s))
    return O.op_gelu_tanh_grad(z)


# ---- graphs ------------------------------------------------------------------------------------------------------------
def some_graph(rng):
    kind = rng.randrange(4)
    dims = [rng.choice((1, 1, 2, 3, 4, 8)) for _ in range(4)]
    dtype, act = rng.choice(("f32", "f32", "bf16")), rng.choice(("none", "silu", "gelu"))
    if kind == 0:
        return group_norm_graph(*dims, dtype, act, rng.choice(("none", "stats", "checkpoint")))
    if kind == 1:
        return group_norm_backward_graph(*dims, dtype, act, rng.choice(("stats", "checkpoint")))
    return (checkpoint_graph if kind == 2 else checkpoint_backward_graph)(*dims[:3], dtype, act, rng.random() < 0.5)


def changed(spec, rng):
    ins, ops, outs = list(spec.inputs), list(spec.ops), list(spec.outputs)
    for _ in range(rng.choice((1, 1, 1, 2, 3))):
        what = rng.randrange(9)
        k, i = rng.randrange(len(ops)), rng.randrange(len(ins))
        o, t = ops[k], ins[i]
        if what <= 2:                                            # an input's extents: one of them, one more or less, in another order, another's
            dims = list(t.dims)
            how = rng.random()
            if how < 0.5:
                dims[rng.randrange(len(dims))] = rng.choice((1, 2, 3, 4, 8))
            elif how < 0.65:
                dims = [1] + dims if len(dims) < 4 else dims[1:]
            elif how < 0.8:
                rng.shuffle(dims)
            else:
                dims = list(rng.choice(ins).dims)
            ins[i] = TensorSpec(t.name, t.dtype, tuple(dims))
        elif what == 3:
            ins[i] = TensorSpec(t.name, rng.choice(("f32", "bf16", "f16", "e4m3")), t.dims)
        elif what == 4:
            j = rng.randrange(len(outs))
            outs[j] = (outs[j][0], rng.choice(("f32", "bf16", "f16", "e4m3")))
            rng.shuffle(outs)
        elif what == 5 and o.opcode in BINARY:
            ops[k] = OpSpec(o.out, o.opcode, o.inputs[::-1], o.attr)
        elif what == 6:                                          # reads another tensor
            operands = list(o.inputs)
            operands[rng.randrange(len(operands))] = rng.choice([t.name for t in ins] + [p.out for p in ops[:k]])
            ops[k] = OpSpec(o.out, o.opcode, tuple(operands), o.attr)
        elif what == 7:
            attr = dict(o.attr)
            if "axis" in attr:
                attr["axis"] = rng.randrange(4)
            if "value" in attr:
                attr["value"] = rng.choice((-attr["value"], 1.0, 0.5, 1 / 240, 1e-3, 0.0, 2.0))
            ops[k] = OpSpec(o.out, o.opcode, o.inputs, attr)
        elif what == 8:                                          # one output more, or one less
            if rng.random() < 0.5 and all(o.out != n for n, _ in outs):
                outs.insert(rng.randrange(len(outs) + 1), (o.out, rng.choice(("f32", "bf16", "e4m3"))))
            elif len(outs) > 1:
                outs.pop(rng.randrange(len(outs)))
    while True:                                                  # without ops and inputs that nothing reads
        read = {n for n, _ in outs} | {n for o in ops for n in o.inputs}
        kept = [o for o in ops if o.out in read]
        if len(kept) == len(ops):
            return GraphSpec("pattern_changed", [t for t in ins if t.name in read], ops, outs)
        ops = kept


# ---- what the kernels compute ------------------------------------------------------------------------------------------
def launches_of(plan):
    found = []
    for line in plan.describe().split("\n"):
        if line.startswith("launch "):
            found.append((line.split()[1], {}))
        slot = re.match(r"\s+ptr(\d+) (\S+)", line)
        if slot:
            found[-1][1][int(slot[1])] = slot[2]
    return found


def computed(spec, plan, values):
    """{output's name in the listing: what the kernel puts there}, of a plan whose first launch has all operands."""
    launches = launches_of(plan)
    kernel, p = launches[0]
    act = re.match(r"\w+<\w+,(\w+)", plan.info["kernel"])[1]
    flat = {f"in{k}": O.to_f64(values[t.name], t.dtype).reshape(-1) for k, t in enumerate(spec.inputs)}
    tensor = {f"in{k}": t for k, t in enumerate(spec.inputs)}
    op = {o.out: o for o in spec.ops}

    def scales(most):   # most * inv_max + tiny, with the graph's constants
        inv_max = next(o for o in spec.ops if o.opcode == "scale" and op[o.inputs[0]].opcode == "reduce_max")
        return most * inv_max.attr["value"] + next(o for o in spec.ops if o.opcode == "add_scalar" and o.inputs[0] == inv_max.out).attr["value"]

    out = {}
    if kernel == "gn_slab":
        x = flat[p[0]].reshape(tensor[p[0]].dims)
        per_channel = x.shape[2:]
        eps = op[next(o for o in spec.ops if o.opcode == "rsqrt").inputs[0]].attr["value"]
        mu = x.mean((1, 3), keepdims=True)
        r = 1 / np.sqrt(((x - mu) ** 2).mean((1, 3), keepdims=True) + eps)
        n = (x - mu) * r
        out = {p[3]: activated(n * flat[p[1]].reshape(per_channel) + flat[p[2]].reshape(per_channel), act), p.get(4): mu, p.get(5): r}
        if 6 in p:
            out[p[7]] = scales(np.abs(n).max((1, 3), keepdims=True))
            out[p[6]] = n / out[p[7]]
    elif kernel == "gn_bwd_slab":
        dy = flat[p[5]].reshape(tensor[p[5]].dims)
        per_group, per_channel = (dy.shape[0], 1, dy.shape[2], 1), dy.shape[2:]
        v, centre, r, gamma = flat[p[0]].reshape(dy.shape), flat[p[1]].reshape(per_group), flat[p[2]].reshape(per_group), flat[p[3]].reshape(per_channel)
        n = v * centre if tensor[p[0]].dtype == "e4m3" else (v - centre) * r
        dz = dy if act == "none" else dy * slope(n * gamma + flat[p[4]].reshape(per_channel), act)
        g = dz * gamma
        out[p[6]] = (g - g.mean((1, 3), keepdims=True) - n * (g * n).mean((1, 3), keepdims=True)) * r
        dbeta, dgamma = (launches[1][1][1], launches[1][1][2]) if len(launches) > 1 else (p[7], p[8])
        out[dbeta], out[dgamma] = dz.sum((0, 1)), (dz * n).sum((0, 1))
    elif kernel in ("checkpoint_wave", "checkpoint_block"):
        z = flat[p[0]].reshape(-1, tensor[p[0]].dims[-1])
        if 1 in p:   # the bias starts over after its own rows
            bias = flat[p[1]].reshape(-1, z.shape[1])
            z = z + bias[np.arange(z.shape[0]) % bias.shape[0]]
        out[p[4]] = scales(np.abs(z).max(1, keepdims=True))
        out[p[3]] = z / out[p[4]]
        if 2 in p:
            out[p[2]] = activated(z, act)
    else:
        assert kernel in ("checkpoint_grad", "checkpoint_grad_sums"), kernel
        z = flat[p[0]].reshape(-1, tensor[p[0]].dims[-1]) * flat[p[1]].reshape(-1, 1)
        out[p[3]] = z if 2 not in p else flat[p[2]].reshape(z.shape) * slope(z, act)
        if kernel == "checkpoint_grad_sums":
            sums = launches[1][1][1] if len(launches) > 1 else p[4]
            out[sums] = out[p[3]]   # (folded by the caller to as many columns as the output has)
    return out


@pytest.mark.parametrize("seed", [1, 2])
def test_what_is_taken_means_what_is_computed(seed):
    rng = random.Random(seed)
    taken = dict.fromkeys(FAMILIES, 0)
    for _ in range(2500):
        spec = changed(some_graph(rng), rng)
        try:
            graph = B.Graph.from_spec(spec)
            plan = B.Plan(graph)
        except (B.FsError, KeyError):   # no graph: extents, types or an axis that do not fit
            continue
        if plan.info["pattern"] not in FAMILIES:
            continue
        whole = [c["candidate"] for c in plan.candidates() if not c["kernel"].startswith(("gn_stats", "gn_bwd_sums"))]
        if not whole:
            continue
        values = {}
        draw = np.random.default_rng(rng.randrange(1 << 30))
        for t in spec.inputs:
            v = draw.uniform(0.5, 1.5, t.dims) if t.dtype == "f32" and t.dims[-1] == 1 else draw.standard_normal(t.dims) + 0.3
            values[t.name] = quantise(v, t.dtype)
        env = O.evaluate(spec, values, keep_all=True)
        got = computed(spec, B.Plan(graph, candidate=rng.choice(whole)), values)
        taken[plan.info["pattern"]] += 1
        for k, (name, dtype) in enumerate(spec.outputs):
            op = next(o for o in spec.ops if o.out == name)
            want = env[op.inputs[0] if op.opcode == "convert" and dtype == "e4m3" else name]   # (before its rounding)
            have = got.get(f"out{k}")
            text = f"{plan.info['kernel']} {name} {spec}"
            assert have is not None, text
            if op.opcode == "reduce_sum" and have.size != want.size:
                have = have.reshape(-1, want.size).sum(0)
            assert have.size == want.size and np.allclose(have.reshape(-1), want.reshape(-1), rtol=1e-6, atol=1e-6, equal_nan=True), text
    assert min(taken.values()) > 100, taken
