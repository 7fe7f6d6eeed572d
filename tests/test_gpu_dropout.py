"""Dropout on the GPU: what is kept is the oracle's to the element, in every form and launch shape, and values are within the bounds of
their arithmetic."""
import numpy as np
import pytest

import workloads as W
from oracle import oracle as O
from paper_2009_10924_amd import binding as B
from tests import operator_bounds as E
from tests.gpu_util import note, run_spec
from workloads.graphs import GraphSpec, OpSpec, TensorSpec, _softmax_ops

pytestmark = pytest.mark.gpu


def _values(spec, inputs):
    return {t.name: O.to_f64(inputs[t.name], t.dtype) for t in spec.inputs}


def _forward_case(rows, cols, p, dtype, act, bias, residual, scheme, seed=1):
    spec = W.dropout_graph(rows, cols, p, dtype=dtype, act=act, bias=bias, residual=residual)
    inputs = W.make_inputs(spec, seed)
    note(f"  case {spec.name} p={p} {scheme}")
    got, _, info, _ = run_spec(spec, inputs, scheme, repeat=2)
    v, ref = _values(spec, inputs), O.evaluate(spec, inputs, keep_all=True)
    z = v["x"] + v["bias"] if bias else v["x"]
    size = np.abs(v["x"]) + (np.abs(v["bias"]) if bias else 0.0)
    scale = 65536.0 / (65536 - round(65536 * p))
    # z's rounding (slopes of the activations are below 1.2), the activation's, the product's, the residual's
    name = spec.outputs[0][0]
    error = scale * (2.0 * E.U32 * size + E.activation_error(z, act) + E.U32 * size) + E.U32 * (np.abs(ref[name]))
    E.close(got[name], ref[name], dtype, error, spec.name)
    if not residual and act == "none" and not bias:
        kept, _ = O.dropout_kept((rows, cols), inputs["state"], p)
        assert np.array_equal(got[name] != 0.0, kept & (v["x"] != 0.0))
    return info


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1), (1, 8), (5, 3), (3, 7), (7, 9), (64, 128), (33, 1000), (2, 4097), (1000, 20)])
def test_kept_elements(shape, dtype):
    for scheme in ("unfused", "auto"):
        for p in (0.1, 0.5):
            info = _forward_case(*shape, p, dtype, "none", False, False, scheme)
    assert info["pattern"] == "dropout"


@pytest.mark.parametrize("p", [0.0, 2.0 ** -16, 0.9, 65535.0 / 65536.0])
def test_probabilities_at_the_ends(p):
    for scheme in ("unfused", "auto"):
        _forward_case(37, 264, p, "f32", "none", False, False, scheme)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
def test_forms(act, dtype):
    for bias in (False, True):
        for residual in (False, True):
            for shape in ((19, 136), (6, 131)):
                _forward_case(*shape, 0.25, dtype, act, bias, residual, "auto")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("cols", [1, 2, 5, 7, 9, 10, 11, 12, 13, 14, 15, 17, 23, 63])
def test_ends_of_rows(cols, dtype):
    """A row's last group holds 1 to 7 elements of its own."""
    _forward_case(300, cols, 0.3, dtype, "none", True, True, "auto")
    _forward_case(300, cols, 0.5, dtype, "none", False, False, "auto")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
@pytest.mark.parametrize("dbias", [False, True])
def test_backward(act, dtype, dbias):
    for rows, cols in ((1, 16), (65, 136), (40, 131), (3, 5)):
        for bias in ((False, True) if act != "none" else (False,)):
            spec = W.dropout_backward_graph(rows, cols, 0.2, dtype=dtype, act=act, bias=bias, dbias=dbias, sequence=7)
            inputs = W.make_inputs(spec, 3)
            note(f"  case {spec.name}")
            v, ref = _values(spec, inputs), O.evaluate(spec, inputs, keep_all=True)
            for scheme in ("unfused", "auto"):
                got, _, info, _ = run_spec(spec, inputs, scheme, repeat=2)
                z = (v["x"] + (v["bias"] if bias else 0.0)) if act != "none" else np.zeros((rows, cols))
                g = np.abs(ref["g"])
                error = g * E.slope_error(z, act) + 3.0 * E.U32 * np.abs(ref[spec.outputs[0][0]]) + g * 2.0 * E.U32
                E.close(got[spec.outputs[0][0]], ref[spec.outputs[0][0]], dtype, error, spec.name)
                if dbias:
                    total = np.abs(ref[spec.outputs[0][0]]).sum(0, keepdims=True)
                    E.close(got["dbias"], ref["dbias"], "f32", error.sum(0, keepdims=True) + E.sum_error(total), spec.name + " dbias")


@pytest.mark.parametrize("ragged", [False, True])
def test_dropped_elements_are_zero_whatever_they_hold(ragged):
    """NaN and infinities count only where they are kept."""
    spec = W.dropout_graph(16, 67 if ragged else 64, 0.5, dtype="f32")
    inputs = W.make_inputs(spec, 5)
    x = inputs["x"]
    x.flat[0::3], x.flat[1::3] = np.nan, np.inf
    kept, _ = O.dropout_kept(x.shape, inputs["state"], 0.5)
    for scheme in ("unfused", "auto"):
        raw = run_spec(spec, inputs, scheme)[1]["d"]
        assert np.array_equal(raw[~kept], np.zeros((~kept).sum(), np.float32))
        assert np.array_equal(np.isnan(raw), kept & np.isnan(x)) and np.array_equal(np.isinf(raw), kept & np.isinf(x))


def _candidates(spec, inputs, compare):
    """Every candidate of the plan (those whose registers do not suffice refuse), and the per-op plan."""
    graph = B.Graph.from_spec(spec)
    n = B.Plan(graph, "auto").info["n_candidates"]
    ran = 0
    for opts in [None] + list(range(n)):
        note(f"  case {spec.name} candidate {opts}")
        try:
            got, raw, info, plan = run_spec(spec, inputs, "unfused") if opts is None else run_spec(spec, inputs, "auto", candidate=opts)
        except B.FsError as e:
            if "scratch memory" in e.text:
                continue
            raise
        compare(got, raw, info, plan)
        ran += 1
    return ran


@pytest.mark.parametrize("dtype,dims", [("f16", (2, 3, 32, 128)), ("f32", (2, 3, 24, 100)), ("f16", (1, 2, 30, 587)), ("bf16", (1, 1, 9, 2359)),
                                        ("bf16", (1, 1, 5, 20000)), ("f32", (1, 1, 3, 66000)), ("bf16", (1, 1, 3, 70001))])
def test_softmax_with_dropout_in_one_kernel(dims, dtype):
    """Attention probabilities: row lengths that end inside a step, lie on the tensor's grid, take a workgroup, and go chunk by chunk."""
    spec = GraphSpec("pattern_softmax_dropout", [TensorSpec("x", dtype, dims), TensorSpec("state", "i32", (4,))],
                     _softmax_ops("x", 3) + [OpSpec("d", "dropout", ("y", "state"), {"probability": 0.25, "sequence": 9})], [("d", dtype)])
    inputs = W.make_inputs(spec, 2)
    ref = O.evaluate(spec, inputs)["d"]

    def compare(got, raw, info, plan):
        # exponent's argument (|x - max| below 16 here), exponential, sum of positive terms, quotient, product
        E.close(got["d"], ref, dtype, np.abs(ref) * E.U32 * (2 * 16.0 + 64.0 + 8.0), f"{spec.name} {info['kernel']}")
        assert np.array_equal(got["d"] != 0.0, ref != 0.0) or dtype != "f32"

    assert _candidates(spec, inputs, compare) >= 2
    assert B.Plan(B.Graph.from_spec(spec)).info["kernel"].startswith("row_generated")


@pytest.mark.parametrize("rows,cols,dtype", [(70, 256, "bf16"), (33, 250, "f32"), (9, 4104, "f16")])
def test_layernorm_behind_a_dropped_branch(rows, cols, dtype):
    """dropout(x + bias) + res through LayerNorm, and two dropouts of one state in one kernel."""
    ops = [OpSpec("z", "add", ("x", "bias")), OpSpec("d", "dropout", ("z", "state"), {"probability": 0.1}), OpSpec("h", "add", ("d", "res")),
           OpSpec("mu", "reduce_mean", ("h",), {"axis": 1}), OpSpec("c", "sub", ("h", "mu")), OpSpec("q", "square", ("c",)),
           OpSpec("v", "reduce_mean", ("q",), {"axis": 1}), OpSpec("ve", "add_scalar", ("v",), {"value": 1e-5}), OpSpec("r", "rsqrt", ("ve",)),
           OpSpec("n", "mul", ("c", "r")), OpSpec("y", "dropout", ("n", "state"), {"probability": 0.5, "sequence": 1})]
    spec = GraphSpec("pattern_dropped_layernorm", [TensorSpec("x", dtype, (rows, cols)), TensorSpec("bias", dtype, (cols,)), TensorSpec("state", "i32", (4,)),
                                                   TensorSpec("res", dtype, (rows, cols))], ops, [("h", dtype), ("y", dtype)])
    inputs = W.make_inputs(spec, 4)
    ref = O.evaluate(spec, inputs, keep_all=True)
    size = 1.2 * (np.abs(O.to_f64(inputs["x"], dtype)) + np.abs(O.to_f64(inputs["bias"], dtype))) + np.abs(O.to_f64(inputs["res"], dtype))
    h_error = 4.0 * E.U32 * size
    top = np.abs(ref["h"]).mean(1, keepdims=True)
    n_error = ref["r"] * (h_error + 64 * E.U32 * top + E.U32 * np.abs(ref["c"])) + 70 * E.U32 * np.abs(ref["n"])

    def compare(got, raw, info, plan):
        E.close(got["h"], ref["h"], dtype, h_error, info["kernel"] + " h")
        E.close(got["y"], ref["y"], dtype, 2.0 * n_error, info["kernel"] + " y")

    assert _candidates(spec, inputs, compare) >= 2


def test_norm_backward_with_dropout_every_shape():
    for dtype, rows, cols, p in (("bf16", 96, 512, 0.1), ("f32", 41, 1001, 0.25), ("f16", 30, 264, 0.0), ("bf16", 1, 4096, 0.1)):
        spec = W.rmsnorm_residual_backward_graph(rows, cols, dtype=dtype, p=p, sequence=3)
        inputs = W.make_inputs(spec, 6)
        ref = O.evaluate(spec, inputs, keep_all=True)
        r = np.abs(ref["r"])
        mean_size = np.abs(ref["gn"]).mean(1, keepdims=True)
        dh_error = r * (4 * E.U32 * np.abs(ref["g"]) + np.abs(ref["nh"]) * (70 * E.U32) * (mean_size + np.abs(ref["m"]))) + 4 * E.U32 * (np.abs(ref["cr"]) + np.abs(ref["dres"]))
        scale = 65536.0 / (65536 - round(65536 * p))

        def compare(got, raw, info, plan):
            E.close(got["dh"], ref["dh"], dtype, dh_error, f"{spec.name} {info['kernel']} dh")
            total = np.abs(ref["dnh"]).sum(0, keepdims=True)
            E.close(got["dgamma"], ref["dgamma"], "f32", E.sum_error(total, 64 + 4), f"{spec.name} {info['kernel']} dgamma")
            if p > 0.0:
                E.close(got["dx"], ref["dx"], dtype, scale * dh_error + E.U32 * np.abs(ref["dx"]), f"{spec.name} {info['kernel']} dx")

        assert _candidates(spec, inputs, compare) >= 2


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sums_over_one_row(dtype):
    """Sums, means and maxima over leading axes of extent 1 are the row's own values, whatever reads them."""
    spec = GraphSpec("pattern_one_row", [TensorSpec("x", dtype, (1, 1, 300)), TensorSpec("state", "i32", (4,)), TensorSpec("g", dtype, (300,))],
                     [OpSpec("d", "dropout", ("x", "state"), {"probability": 0.5}), OpSpec("a", "reduce_sum", ("d",), {"axis": 0}),
                      OpSpec("b", "reduce_mean", ("a",), {"axis": 0}), OpSpec("m", "reduce_max", ("d",), {"axis": 1}),
                      OpSpec("y", "mul", ("b", "g"))], [("d", dtype), ("b", "f32"), ("m", "f32"), ("y", dtype)])
    inputs = W.make_inputs(spec, 8)
    ref = O.evaluate(spec, inputs, keep_all=True)

    def compare(got, raw, info, plan):
        for name, dt in spec.outputs:
            E.close(got[name], ref[name].reshape(got[name].shape), dt, 2 * E.U32 * np.abs(ref[name]).reshape(got[name].shape), f"{info['kernel']} {name}")

    assert _candidates(spec, inputs, compare) >= 2


def test_transposed_and_stretched_neighbours():
    """A dropout behind a folded transpose goes by its own rows; one of a value that stretches later is drawn once."""
    dims = (2, 5, 3, 16)
    spec = GraphSpec("pattern_dropped_view", [TensorSpec("x", "f32", dims), TensorSpec("state", "i32", (4,)), TensorSpec("gain", "f32", (16,))],
                     [OpSpec("t", "transpose", ("x",), {"perm": (0, 2, 1, 3)}), OpSpec("d", "dropout", ("t", "state"), {"probability": 0.5}),
                      OpSpec("y", "mul", ("d", "gain"))], [("y", "f32")])
    inputs = W.make_inputs(spec, 1)
    ref = O.evaluate(spec, inputs)["y"]
    for scheme in ("unfused", "auto"):
        got, _, info, _ = run_spec(spec, inputs, scheme)
        E.close(got["y"], ref, "f32", 3 * E.U32 * np.abs(ref), scheme)
    spec = GraphSpec("pattern_stretched_drop", [TensorSpec("g", "f32", (5, 1)), TensorSpec("state", "i32", (4,)), TensorSpec("x", "f32", (5, 32))],
                     [OpSpec("d", "dropout", ("g", "state"), {"probability": 0.5}), OpSpec("y", "mul", ("x", "d"))], [("y", "f32")])
    inputs = W.make_inputs(spec, 1)
    ref = O.evaluate(spec, inputs)["y"]
    got, _, info, _ = run_spec(spec, inputs)
    E.close(got["y"], ref, "f32", 3 * E.U32 * np.abs(ref), "stretched")


def test_in_place():
    """The element-wise kernel may write over its input or residual."""
    import torch
    for cols in (64, 67, 7, 9, 15, 654):
        spec = W.dropout_graph(50, cols, 0.3, dtype="bf16", residual=True, bias=True)
        inputs = W.make_inputs(spec, 2)
        want = run_spec(spec, inputs)[1]["y"]
        plan = B.Plan(B.Graph.from_spec(spec))
        for over in ("x", "res"):
            dev = {t.name: B.to_device(inputs[t.name], t.dtype) for t in spec.inputs}
            plan.execute([dev[t.name] for t in spec.inputs], [dev[over]])
            torch.cuda.synchronize()
            assert np.array_equal(B.to_host(dev[over], "bf16"), want), (cols, over)


def test_a_captured_graph_draws_anew():
    """The state is read when the kernel runs: a replay after the offset has moved gives the new draw, every time as the eager call does."""
    import torch
    for spec in (W.dropout_graph(64, 131, 0.5, dtype="f32", residual=True), W.dropout_backward_graph(96, 264, 0.5, dtype="f32", act="gelu")):
        inputs = W.make_inputs(spec, 2)
        plan = B.Plan(B.Graph.from_spec(spec))
        ws = plan.make_workspace()
        dev = {t.name: B.to_device(inputs[t.name], t.dtype) for t in spec.inputs}
        ins = [dev[t.name] for t in spec.inputs]
        outs, eager = B.alloc_outputs(spec), B.alloc_outputs(spec)
        plan.execute(ins, outs, ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            plan.execute(ins, outs, ws)
        seen = []
        for step in range(3):
            dev["state"][2] += 1
            for t in outs:
                t.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            plan.execute(ins, eager, ws)
            torch.cuda.synchronize()
            for a, b in zip(outs, eager):
                assert torch.equal(a, b)
            seen.append(outs[0].clone())
        assert not torch.equal(seen[0], seen[1]) and not torch.equal(seen[1], seen[2])


def test_another_stream_and_sequences_of_their_own():
    import torch
    draws = []
    side = torch.cuda.Stream()
    for sequence in (0, 1, 0xFFFFFFFF):
        spec = W.dropout_graph(128, 256, 0.5, dtype="f32", sequence=sequence)
        inputs = W.make_inputs(spec, 2)
        plan = B.Plan(B.Graph.from_spec(spec))
        ins, outs = [B.to_device(inputs[t.name], t.dtype) for t in spec.inputs], B.alloc_outputs(spec)
        torch.cuda.synchronize()
        plan.execute(ins, outs, stream=side.cuda_stream)
        side.synchronize()
        kept, _ = O.dropout_kept((128, 256), inputs["state"], 0.5, sequence)
        assert np.array_equal(outs[0].cpu().numpy() != 0.0, kept)
        draws.append(kept)
    # neighbouring sequences share no more than chance lets them: half of 32768, give or take six standard deviations of 90
    assert abs(int((draws[0] == draws[1]).sum()) - 16384) < 6 * 91


def test_packed_with_others():
    """Softmax with dropout beside a normalisation in one packed launch."""
    from tests.gpu_util import run_pack
    specs = [GraphSpec("pattern_softmax_dropout", [TensorSpec("x", "f32", (24, 96)), TensorSpec("state", "i32", (4,))],
                       _softmax_ops("x", 1) + [OpSpec("d", "dropout", ("y", "state"), {"probability": 0.25, "sequence": k})], [("d", "f32")]) for k in range(3)]
    specs.append(W.log_softmax_graph(16, 64))
    inputs = [W.make_inputs(s, k) for k, s in enumerate(specs)]
    outs, info = run_pack(specs, inputs)
    for s, i, o in zip(specs[:3], inputs, outs):
        ref = O.evaluate(s, i)["d"]
        E.close(o["d"], ref, "f32", np.abs(ref) * E.U32 * 104.0, s.name)
    assert info["n_kernels"] == 1
