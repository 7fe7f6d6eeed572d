"""Group normalisation and 8-bit checkpoints as they are used: a residual branch forward and backward between its matrix products,
replayed from a graph, on two streams at once, from the static scratch array, at the limit of 2^31 elements, on values that are not
finite, and the gradients against those without a checkpoint.  Bounds are those of the patterns' own tests."""
import numpy as np
import pytest

from oracle import oracle as O
from paper_2009_10924_amd import binding as B
from workloads import (checkpoint_backward_graph, checkpoint_graph, checkpointed_block_graph, group_norm_backward_graph, group_norm_graph, make_inputs,
                       quantise)

from .gpu_util import note, run_spec
from .test_gpu_checkpoint import EPS, bounds, within
from .test_gpu_group_norm import U, backward_bounds, every_candidate, forward_bounds

pytestmark = pytest.mark.gpu


def parts_of(batch, positions, groups, dim, hidden, block, dtype, act):
    rows = batch * positions
    return [("f1_", group_norm_graph(batch, positions, groups, dim, dtype, act, "checkpoint"), {}),
            ("f2_", checkpoint_graph(rows, hidden // block, block, dtype, "gelu", True), {}),
            ("b2_", checkpoint_backward_graph(rows, hidden // block, block, dtype, "gelu", True), {"q": "f2_q", "s": "f2_s"}),
            ("b1_", group_norm_backward_graph(batch, positions, groups, dim, dtype, act, "checkpoint"),
             {"q": "f1_q", "s": "f1_s", "r": "f1_r", "gamma": "f1_gamma", "beta": "f1_beta"})]


def clear(tensors):
    """Bytes that are NaN in every floating type and no state a kernel may rely on."""
    import torch
    for t in tensors:
        t.view(torch.uint8).fill_(0xFF)


def product(a, w):
    """The matrix product between two stages: in float32, stored in the type of `a`."""
    return (a.float().reshape(-1, w.shape[0]) @ w).to(a.dtype)


@pytest.mark.parametrize("sizes", [(2, 64, 4, 16, 256, 64, "bf16", "silu"), (3, 50, 5, 7, 100, 50, "f32", "gelu"), (1, 1000, 8, 40, 640, 128, "f16", "silu"),
                                   (2, 4000, 32, 10, 256, 32, "bf16", "gelu")], ids=lambda s: "x".join(map(str, s)))
def test_block_between_its_products(sizes):
    """Stage by stage, the products in between; every stage's outputs against the oracle on what that stage read."""
    import torch
    batch, positions, groups, dim, hidden, block, dtype, act = sizes
    channels = groups * dim
    spec = checkpointed_block_graph(*sizes)
    inp = make_inputs(spec, seed=1)
    dev = {t.name: B.to_device(inp[t.name], t.dtype) for t in spec.inputs}
    out = dict(zip([n for n, _ in spec.outputs], B.alloc_outputs(spec)))
    clear(list(out.values()))
    clear([dev[dst] for _, dst in spec.external])                                   # not there yet
    prog = B.Program(B.Graph.from_spec(spec))
    assert prog.info["n_stages"] == 4
    ws = prog.make_workspace()
    clear([ws])
    ins, outs = [dev[t.name].data_ptr() for t in spec.inputs], [out[n].data_ptr() for n, _ in spec.outputs]
    gen = torch.Generator(device="cuda").manual_seed(3)
    w1 = torch.randn(channels, hidden, device="cuda", generator=gen) / channels ** 0.5
    w2 = torch.randn(hidden, hidden, device="cuda", generator=gen) / hidden ** 0.5
    stream = torch.cuda.current_stream().cuda_stream
    for stage in range(4):
        prog.bind_stage(stage, ins, outs, ws.data_ptr(), ws.numel(), stream)()
        if stage == 0:
            dev["f2_x"].copy_(product(out["f1_y"], w1).view_as(dev["f2_x"]))
        elif stage == 1:
            dev["b2_dy"].copy_(product(out["f2_y"], w2).view_as(dev["b2_dy"]))       # (the rest of the network)
        elif stage == 2:
            dev["b1_dy"].copy_(product(out["b2_dx"], w1.t().contiguous()).view_as(dev["b1_dy"]))
    torch.cuda.synchronize()
    host = {t.name: B.to_host(dev[t.name], t.dtype) for t in spec.inputs}
    host.update({n: B.to_host(out[n], d) for n, d in spec.outputs})
    for prefix, part, shared in parts_of(*sizes):
        read = {t.name: host[shared.get(t.name, prefix + t.name)] for t in part.inputs}
        env = O.evaluate(part, read, keep_all=True)
        if prefix == "f1_":
            allowed = forward_bounds(part, env, act, dtype)
        elif prefix == "b1_":
            allowed = backward_bounds(env, dtype)
        else:
            env = O.evaluate(part, read)      # (q before it is rounded)
            allowed = bounds(part, read, env, dtype)
        for name, d in part.outputs:
            want = env["q_d"] if name == "q" and prefix == "f1_" else env[name]
            within(O.to_f64(host[prefix + name], d).reshape(want.shape), want, allowed[name], f"{spec.name}/{prefix}{name}")


def family_specs(dtype):
    """One graph per kind of launch: a slab, statistics and apply, one with a launch in between; a fold; several entries a workgroup."""
    return [group_norm_graph(2, 100, 8, 16, dtype, "silu", "checkpoint"), group_norm_graph(2, 9000, 4, 10, dtype, "gelu", "checkpoint"),
            group_norm_graph(1, 60000, 32, 8, dtype, "silu", "stats"), group_norm_backward_graph(3, 197, 5, 7, dtype, "gelu", "stats"),
            group_norm_backward_graph(2, 9000, 4, 10, dtype, "silu", "checkpoint"), group_norm_backward_graph(1, 60000, 32, 8, dtype, "silu", "checkpoint"),
            group_norm_backward_graph(20000, 1, 2, 4, dtype, "silu", "stats"), checkpoint_graph(300, 4, 32, dtype, "gelu", True),
            checkpoint_graph(5, 1, 70001, dtype, "silu", False), checkpoint_backward_graph(1000, 1, 520, dtype, "gelu", True),
            checkpoint_backward_graph(100, 3, 77, dtype, "none")]


def ready(spec, seed=0):
    inp = make_inputs(spec, seed=seed)
    plan = B.Plan(B.Graph.from_spec(spec))
    ins, outs, ws = [B.to_device(inp[t.name], t.dtype) for t in spec.inputs], B.alloc_outputs(spec), plan.make_workspace()
    assert plan.info["pattern"] != "unfused"

    def call(stream):
        plan.bind([t.data_ptr() for t in ins], [t.data_ptr() for t in outs], ws.data_ptr() if ws is not None else 0, ws.numel() if ws is not None else 0, stream)()
    return plan, ins, outs, ws, call


def raw(t):
    import torch
    return t.view(torch.uint8).clone()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_replayed_from_one_graph(dtype):
    """All of them captured one after another into one graph; every replay equals the eager run bit for bit, with eager calls of the
    same plans (on workspaces of their own) between the replays."""
    import torch
    runs = [ready(s, seed=k) for k, s in enumerate(family_specs(dtype))]
    eager = [ready(s, seed=k) for k, s in enumerate(family_specs(dtype))]
    now = torch.cuda.current_stream().cuda_stream
    for r in eager:
        r[4](now)
    torch.cuda.synchronize()
    want = [[raw(t) for t in r[2]] for r in eager]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for r in runs:
            r[4](torch.cuda.current_stream().cuda_stream)
    for replay in range(3):
        clear([t for r in runs for t in r[2]] + [r[3] for r in runs if r[3] is not None])
        for r in eager:
            r[4](now)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for r, e, ref in zip(runs, eager, want):
            for t, u, v in zip(r[2], e[2], ref):
                assert torch.equal(raw(t), v) and torch.equal(raw(u), v), f"replay {replay} {r[0].info['kernel']}"


def test_two_streams_at_once():
    """The same plans on two streams, each with its own outputs and workspaces, 20 times without waiting for each other."""
    import torch
    specs = family_specs("f16")
    first, second = [ready(s, seed=k) for k, s in enumerate(specs)], [ready(s, seed=k) for k, s in enumerate(specs)]
    for r in first:
        r[4](torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    want = [[raw(t) for t in r[2]] for r in first]
    clear([t for r in first + second for t in r[2]])
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for k in range(20):
        for a, b in zip(first, second[::-1]):
            a[4](streams[0].cuda_stream)
            b[4](streams[1].cuda_stream)
    torch.cuda.synchronize()
    for runs in (first, second):
        for r, ref in zip(runs, want):
            assert all(torch.equal(raw(t), v) for t, v in zip(r[2], ref)), r[0].info["kernel"]


def test_static_scratch_gives_the_same():
    import torch
    for k, spec in enumerate(family_specs("bf16")):
        plan, ins, outs, ws, call = ready(spec, seed=k)
        stream = torch.cuda.current_stream().cuda_stream
        call(stream)
        torch.cuda.synchronize()
        want = [raw(t) for t in outs]
        clear(outs)
        assert plan.info["workspace_bytes"] <= B.FS_STATIC_SCRATCH_BYTES
        plan.execute_static_ptrs([t.data_ptr() for t in ins], [t.data_ptr() for t in outs], stream)
        torch.cuda.synchronize()
        assert all(torch.equal(raw(t), v) for t, v in zip(outs, want)), plan.info["kernel"]
        with pytest.raises(B.FsError, match="shares memory"):
            plan.execute_static_ptrs([t.data_ptr() for t in ins], [ins[0].data_ptr()] + [t.data_ptr() for t in outs[1:]], stream)


def test_nothing_is_written_beside_the_outputs():
    """Outputs as parts of larger buffers: the bytes in front of and behind each stay as they were."""
    import torch
    for dtype in ("bf16", "f32"):
        for k, spec in enumerate(family_specs(dtype) + [checkpoint_graph(7, 3, 100, dtype, "silu", True), group_norm_graph(3, 7, 3, 5, dtype, "gelu", "checkpoint")]):
            inp = make_inputs(spec, seed=k)
            plan = B.Plan(B.Graph.from_spec(spec))
            ins, ws = [B.to_device(inp[t.name], t.dtype) for t in spec.inputs], plan.make_workspace()
            outs = B.alloc_outputs(spec)
            wide = [torch.full((512 + t.numel() * t.element_size() + 512,), 0xA5, dtype=torch.uint8, device="cuda") for t in outs]
            plan.bind([t.data_ptr() for t in ins], [w.data_ptr() + 512 for w in wide], ws.data_ptr() if ws is not None else 0, ws.numel() if ws is not None else 0,
                      torch.cuda.current_stream().cuda_stream)()
            torch.cuda.synchronize()
            for w, t in zip(wide, outs):
                assert bool((w[:512] == 0xA5).all()) and bool((w[512 + t.numel() * t.element_size():] == 0xA5).all()), plan.info["kernel"]


# ---- values that make it hard ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("shape", [(2, 60, 4, 8), (2, 5000, 4, 10), (1, 60000, 32, 8), (9000, 2, 4, 3)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_groups_do_not_see_each_other(shape, dtype):
    """One value of one group not finite: that group is, the others and their sums are to the bit what they were."""
    batch, positions, groups, dim = shape
    for poison in (np.nan, np.inf, -np.inf):
        spec = group_norm_graph(*shape, dtype=dtype, act="silu", keep="checkpoint")
        inp = make_inputs(spec, seed=2)
        clean, _, info, _ = run_spec(spec, inp)
        x = O.to_f64(inp["x"], dtype).copy()
        x[batch - 1, positions // 2, 1, dim - 1] = poison
        got, _, _, _ = run_spec(spec, {**inp, "x": quantise(x, dtype)})
        for name, _ in spec.outputs:
            a, b = got[name].copy(), clean[name].copy()
            ill = a[batch - 1, :, 1]
            if name in ("y", "q"):                    # a NaN everywhere, or (an infinity) a NaN where it is and at least no number like before
                assert np.isnan(ill[positions // 2, dim - 1]) and np.isnan(ill).all() or name == "q", (info["kernel"], name)
            a[batch - 1, :, 1] = b[batch - 1, :, 1] = 0
            assert np.array_equal(a, b), (info["kernel"], name, poison)
        spec = group_norm_backward_graph(*shape, dtype=dtype, act="gelu", keep="stats")
        inp = make_inputs(spec, seed=2)
        clean, _, info, _ = run_spec(spec, inp)
        dy = O.to_f64(inp["dy"], dtype).copy()
        dy[batch - 1, positions // 2, 1, dim - 1] = poison
        got, _, _, _ = run_spec(spec, {**inp, "dy": quantise(dy, dtype)})
        assert not np.isfinite(got["dx"][batch - 1, positions // 2, 1, dim - 1])
        got["dx"][batch - 1, :, 1] = clean["dx"][batch - 1, :, 1] = 0
        assert np.array_equal(got["dx"], clean["dx"]), (info["kernel"], poison)
        for name in ("dgamma", "dbeta"):
            a, b = got[name].reshape(groups, dim), clean[name].reshape(groups, dim)
            assert not np.isfinite(a[1, dim - 1]), (info["kernel"], name)
            a[1, dim - 1] = b[1, dim - 1] = 0
            assert np.array_equal(a, b), (info["kernel"], name)


@pytest.mark.parametrize("shape", [(2, 60, 4, 8), (2, 5000, 4, 10), (1, 3, 2, 2)], ids=lambda s: "x".join(map(str, s)))
def test_groups_far_from_zero_and_without_spread(shape):
    """A mean of a thousand deviations, groups of one value, of zeros, of very large values.  A mean off by dm adds dm^2 to the
    variance, half of (dm r)^2 relative to r: no part of the other tests' bounds, where means are small."""
    for k, (base, spread) in enumerate([(1000.0, 1.0), (-3.0, 0.0), (0.0, 0.0), (1e17, 1e16)]):
        spec = group_norm_graph(*shape, dtype="f32", act="none", keep="checkpoint")
        inp = make_inputs(spec, seed=k)
        noise = np.random.default_rng(k).standard_normal(shape)
        inp["x"] = quantise(base + spread * noise, "f32")
        env = O.evaluate(spec, inp, keep_all=True)
        allowed = forward_bounds(spec, env, "none", "f32")
        more = 0.5 * (100 * U * np.abs(env["x"]).mean((1, 3), keepdims=True) * env["r"]) ** 2
        allowed["r"] = allowed["r"] + more * env["r"]
        allowed["s"] = allowed["s"] + more * env["s"]
        allowed["q"] = allowed["q"] + 2 * more * np.abs(env["q_d"])
        allowed["z"] = allowed["z"] + 1.13 * more * np.abs(env["ng"])
        every_candidate(spec, inp, allowed, env)


def test_checkpoint_of_a_nan_restores_a_nan_there_alone():
    for act, dbias in (("none", False), ("gelu", True), ("silu", False)):
        spec = checkpoint_backward_graph(300, 2, 50, dtype="bf16", act=act, dbias=dbias)
        inp = make_inputs(spec, seed=1)
        clean, _, info, _ = run_spec(spec, inp)
        inp["q"] = inp["q"].copy()
        inp["q"][17, 1, 9] = 0x7F
        inp["q"][18, 0, 3] = 0xFF
        got, _, _, _ = run_spec(spec, inp)
        for name, _ in spec.outputs:
            places = [(0, 1, 9), (0, 0, 3)] if name == "dbias" else [(17, 1, 9), (18, 0, 3)]
            for at in places:
                assert np.isnan(got[name].reshape(clean[name].shape)[at]), (act, name)
                got[name].reshape(clean[name].shape)[at] = clean[name][at] = 0
            assert np.array_equal(got[name], clean[name]), (act, name)


@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("size", [1e3, 1e15, 1e25, 1e35])
def test_slopes_of_very_large_values_are_zero_and_one(act, size):
    """dx = dy act'(q s) for q s up to 448 `size`, whose square is no float32."""
    for dbias in (False, True):
        spec = checkpoint_backward_graph(40, 2, 24, "f32", act, dbias)
        inp = make_inputs(spec, seed=3)
        inp["s"] = np.full_like(inp["s"], size)
        with np.errstate(over="ignore"):
            ref = O.evaluate(spec, inp)
        got, _, info, _ = run_spec(spec, inp)
        assert info["pattern"] == "checkpoint_backward"
        for name, _ in spec.outputs:
            within(got[name], ref[name], bounds(spec, inp, ref, "f32")[name], f"{info['kernel']}/{name}")


@pytest.mark.parametrize("eps", [1e-5, 1e-15, 1e-18])
def test_checkpoint_of_groups_of_zeros_is_zero(eps):
    """1 / sqrt(eps) and the scale's reciprocal are as large as can be there: 0 all the same, in the kernels and where they are not taken."""
    for shape in ((2, 40, 4, 8), (2, 40, 4, 7), (1, 9000, 2, 8)):
        spec = group_norm_graph(*shape, dtype="bf16", act="none", keep="checkpoint", eps=eps)
        inp = make_inputs(spec, seed=1)
        inp["x"] = quantise(np.zeros(shape), "bf16")
        for opts in [{"candidate": i} for i in range(B.Plan(B.Graph.from_spec(spec)).info["n_candidates"])]:
            got, _, info, _ = run_spec(spec, inp, **opts)
            assert not got["q"].any() and np.isfinite(got["s"]).all(), info["kernel"]
            assert np.array_equal(got["z"], np.broadcast_to(O.to_f64(inp["beta"], "bf16"), shape)), info["kernel"]


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_gradient_through_a_checkpoint_stays_near_the_exact_one(act):
    """What the 8 bits cost a gradient: z is off by at most 2^-4 |z| (2^-10 s near zero), and the slope changes by at most
    max |act''| = 0.8 (0.5 for SiLU) times that; the sum over rows by the sum of these."""
    rows, blocks, block = 700, 6, 64
    z_spec = checkpoint_graph(rows, blocks, block, "f32", act, True)
    inp = make_inputs(z_spec, seed=4)
    kept, bits, _, _ = run_spec(z_spec, inp)
    spec = checkpoint_backward_graph(rows, blocks, block, "f32", act, True)
    dy = np.random.default_rng(5).standard_normal((rows, blocks, block)).astype(np.float32)
    got, _, info, _ = run_spec(spec, {"q": quantise(kept["q"], "e4m3"), "s": kept["s"].astype(np.float32), "dy": dy})
    z = inp["x"].astype(np.float64) + inp["bias"].astype(np.float64)
    slope = O.op_gelu_tanh_grad(z) if act == "gelu" else (lambda s: s * (1 + z * (1 - s)))(O.op_sigmoid(z))
    exact = dy * slope
    off = np.abs(dy) * ({"gelu": 0.85, "silu": 0.5}[act] * np.maximum(2.0 ** -4 * np.abs(z), 2.0 ** -10 * kept["s"]) * (1 + 1e-5) + 1e-5)
    within(got["dx"], exact, off + EPS["f32"] * np.abs(exact), "dx")
    within(got["dbias"], exact.sum(0, keepdims=True), off.sum(0, keepdims=True) + 1.6e-5 * np.abs(dy).sum(0, keepdims=True), "dbias")


@pytest.mark.parametrize("shape", [(20000, 1, 2, 4), (9000, 3, 8, 8), (1, 60000, 32, 8), (300, 1, 1, 1)], ids=lambda s: "x".join(map(str, s)))
def test_very_many_entries_and_very_long_ones(shape):
    """Several batch entries per workgroup, and statistics that a launch of their own joins: every candidate."""
    for dtype in ("bf16", "f32"):
        spec = group_norm_graph(*shape, dtype=dtype, act="silu", keep="checkpoint")
        inp = make_inputs(spec, seed=7)
        env = O.evaluate(spec, inp, keep_all=True)
        every_candidate(spec, inp, forward_bounds(spec, env, "silu", dtype), env, unfused=False, repeat=1)
        spec = group_norm_backward_graph(*shape, dtype=dtype, act="silu", keep="checkpoint")
        inp = make_inputs(spec, seed=7)
        env = O.evaluate(spec, inp, keep_all=True)
        every_candidate(spec, inp, backward_bounds(env, dtype), env, unfused=False, repeat=1)


# ---- the largest tensors ---------------------------------------------------------------------------------------------------
def run_repeated(big, small, grows, repeats):
    """`big` is `small` with the tensors in `grows` repeated along the axis where they differ: runs `big` on the repeated inputs of
    `small`; hands back the latter and the outputs, on the device."""
    import torch
    inp = make_inputs(small, seed=6)
    dev = []
    for t, u in zip(small.inputs, big.inputs):
        d = B.to_device(inp[t.name], t.dtype)
        axis = [k for k in range(len(t.dims)) if t.dims[k] != u.dims[k]]
        if axis:
            ones = [1] * len(t.dims)
            ones[axis[0]] = repeats
            d = d.view(torch.uint8).view(*t.dims[:-1], -1).repeat(*ones).view(d.dtype).contiguous()
        assert tuple(d.shape) == tuple(u.dims) and (t.name in grows) == bool(axis)
        dev.append(d)
    plan = B.Plan(B.Graph.from_spec(big))
    assert plan.info["pattern"] != "unfused"
    note(f"  case {big.name} {plan.info['kernel']}")
    outs = B.alloc_outputs(big)
    clear(outs)
    plan.execute(dev, outs, plan.make_workspace())
    torch.cuda.synchronize()
    return inp, {n: o for (n, _), o in zip(big.outputs, outs)}


def check_grown(out, name, dtype, ref, allowed, axis, repeats, what):
    """Every repeat of `out` along `axis`, on the device."""
    import torch
    period = ref.shape[axis]
    want, bound = torch.from_numpy(np.ascontiguousarray(ref)).cuda(), torch.from_numpy(np.array(np.broadcast_to(allowed, ref.shape))).cuda()
    ones = [1] * ref.ndim
    at = 0
    some = max(1, (1 << 26) // ref.size)
    while at < repeats:
        k = min(some, repeats - at)
        got = out.narrow(axis, at * period, k * period)
        if dtype == "e4m3":
            got = got.contiguous().to(torch.float32)
        ones[axis] = k
        over = ((got.double() - want.repeat(*ones)).abs() - bound.repeat(*ones)).max().item()
        assert over <= 0, f"{what}/{name}: repeats {at}..{at + k}: {over:.3e} above the bound"
        at += k


@pytest.mark.parametrize("axis", [0, 1])
def test_group_norm_at_the_element_limit(axis):
    """2^31 - 1048576 values, in 524032 short batch entries or one long one (whose statistics are those of its repeated part; sums of up to
    65536 / 64 more additions in a row than in the small tests: 2000 u instead of 100 u)."""
    act, dtype = "silu", "bf16"
    small_shape, repeats = ((64, 16, 32, 8), 8188) if axis == 0 else ((1, 4096, 32, 8), 2047)
    shape = tuple(n * repeats if k == axis else n for k, n in enumerate(small_shape))
    small, big = (group_norm_graph(*s, dtype=dtype, act=act, keep="checkpoint") for s in (small_shape, shape))
    inp, out = run_repeated(big, small, {"x"}, repeats)
    env = O.evaluate(small, inp, keep_all=True)
    allowed = forward_bounds(small, env, act, dtype)
    more = 1 if axis == 0 else 20
    dn = more * (100 * U * np.abs(env["x"]).mean((1, 3), keepdims=True) * env["r"] + 1e-5 * np.abs(env["n"]))
    for name, d in small.outputs:
        ref = env["q_d"] if name == "q" else env[name]
        bound = allowed[name] * more if name in ("s", "r") else allowed[name] + (2 * dn / env["s"] if name == "q" else 1.13 * dn * np.abs(env["gamma"]) * (1 + EPS[dtype]))
        check_grown(out[name], name, d, ref, bound, axis if ref.shape[axis] > 1 else 0, repeats if out[name].shape != ref.shape else 1, big.name)


@pytest.mark.parametrize("axis", [0, 1])
def test_group_norm_backward_at_the_element_limit(axis):
    act, dtype = "silu", "bf16"
    small_shape, repeats = ((64, 16, 32, 8), 8188) if axis == 0 else ((1, 4096, 32, 8), 2047)
    shape = tuple(n * repeats if k == axis else n for k, n in enumerate(small_shape))
    keep = "checkpoint" if axis == 0 else "stats"
    small, big = (group_norm_backward_graph(*s, dtype=dtype, act=act, keep=keep) for s in (small_shape, shape))
    grows = {"q", "s", "dy", "r"} if axis == 0 else {"x", "dy"}
    inp, out = run_repeated(big, small, grows, repeats)
    env = O.evaluate(small, inp, keep_all=True)
    allowed = backward_bounds(env, dtype)
    more = 1 if axis == 0 else 20
    check_grown(out["dx"], "dx", dtype, env["dx"], allowed["dx"] * more, axis, repeats, big.name)
    for name in ("dgamma", "dbeta"):
        # up to 4096 additions in a row (entries of a workgroup, or positions of a chunk), then folds: 4096 u = 2.5e-4 of the terms
        terms = np.abs(env["dz"] * env["n"] if name == "dgamma" else env["dz"]).sum((0, 1), keepdims=True) * repeats
        within(out[name].double().cpu().numpy().reshape(env[name].shape), env[name] * repeats, 3e-4 * terms + 1.6e-5 * terms, f"{big.name}/{name}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_checkpoints_at_the_element_limit(dtype):
    import torch
    repeats = 4094
    small, big = (checkpoint_graph(n, 16, 64, dtype, "gelu", True) for n in (512, 512 * repeats))
    inp, out = run_repeated(big, small, {"x"}, repeats)
    ref = O.evaluate(small, inp)
    allowed = bounds(small, inp, ref, dtype)
    for name, d in small.outputs:
        check_grown(out[name], name, d, ref[name], allowed[name], 0, repeats, big.name)
    del out
    torch.cuda.empty_cache()
    for act, dbias in (("gelu", True), ("none", False)):
        small, big = (checkpoint_backward_graph(n, 16, 64, dtype, act, dbias) for n in (512, 512 * repeats))
        inp, out = run_repeated(big, small, {"q", "s", "dy"} & {t.name for t in small.inputs}, repeats)
        ref = O.evaluate(small, inp)
        allowed = bounds(small, inp, ref, dtype)
        name = small.outputs[0][0]
        check_grown(out[name], name, dtype, ref[name], allowed[name], 0, repeats, big.name)
        if dbias:
            # 2096128 rows over 768 workgroups of 4 wavefronts: 683 additions in a row, then folds of 12 and 64
            terms = np.abs(O.to_f64(inp["dy"], dtype)).sum(0, keepdims=True) * repeats
            within(out["dbias"].double().cpu().numpy().reshape(ref["dbias"].shape), ref["dbias"] * repeats, (760 * U + 1e-5) * 1.13 * terms, f"{big.name}/dbias")
        del out
        torch.cuda.empty_cache()
