"""Dropout, the 8-bit norm and rotary positions together, as one explored program of a decoder block, whole and stage by stage."""
import numpy as np
import pytest

import workloads as W
from oracle import oracle as O
from paper_2009_10924_amd import binding as B
from tests import operator_bounds as E
from tests.gpu_util import note

pytestmark = pytest.mark.gpu


def _check(spec, inputs, raw, dtype):
    got = {n: O.to_f64(raw[n], d) for n, d in spec.outputs}
    ref = O.evaluate(spec, inputs, keep_all=True, stored={n: got[n] for n in ("b_h",)} if dtype != "f32" else None)
    own = O.evaluate(spec, inputs, keep_all=True)
    scale = 65536.0 / (65536 - round(65536 * 0.1))
    size = scale * (np.abs(ref["attn_out"]) + np.abs(ref["bias_o"])) + np.abs(ref["x"])
    E.close(got["b_h"], own["b_h0"], dtype, 4.0 * E.U32 * size, "b_h")
    for p, h, gain in (("a_", ref["x"], ref["gamma1"]), ("b_", ref["b_h"], ref["gamma2"])):
        E.close(got[p + "r"], ref[p + "r"], "f32", 48.0 * E.U32 * ref[p + "r"] + (4.0 * E.U32 * ref[p + "r"] if dtype == "f32" else 0.0), p + "r")
        n_error = 56.0 * E.U32 * np.abs(ref[p + "n"]) + (ref[p + "r"] * np.abs(gain) * 4.0 * E.U32 * size if dtype == "f32" else 0.0)
        E.close(got[p + "s"], ref[p + "s"], "f32", n_error.max(1, keepdims=True) / 448.0 + 3.0 * E.U32 * ref[p + "s"], p + "s")
        E.eight_bit(got[p + "q"], got[p + "s"], ref[p + "n"], n_error, p + "q")
    for n, lin in (("qs", "q_lin"), ("ks", "k_lin")):
        a = ref[lin]
        half = a.shape[-1] // 2
        both = np.abs(a[..., :half]) + np.abs(a[..., half:])
        E.close(got[n], O.evaluate(spec, inputs, keep_all=True)[n[0] + "r"].transpose(0, 2, 1, 3), dtype,
                (np.concatenate([both, both], -1) * 6.0 * E.U32).transpose(0, 2, 1, 3), n)
    gate = np.abs(ref["ga"]) + E.activation_error(ref["gate"], "silu") / E.U32 / 8.0
    E.close(got["gd"], ref["gd"], dtype, scale * np.abs(ref["up"]) * 8.0 * E.U32 * gate, "gd")
    h_error = 0.0 if dtype != "f32" else 4.0 * E.U32 * size
    E.close(got["y"], ref["y"], dtype, 2.0 * E.U32 * (np.abs(ref["fd"]) + np.abs(ref["b_h"])) + h_error, "y")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sizes", [dict(batch=2, seq=40, heads=8, kv_heads=2, dim=32, ffn=264, sections=(4, 6, 6)),
                                   dict(batch=3, seq=1, heads=3, kv_heads=1, dim=20, ffn=70, sections=(9,))])
def test_decoder_block(sizes, dtype):
    import torch
    spec = W.decoder_block_graph(dtype=dtype, **sizes)
    inputs = W.make_inputs(spec, 4)
    program = B.Program(B.Graph.from_spec(spec))
    note(program.describe())
    kinds = [p["info"]["pattern"] for p in program.patterns()]
    assert program.info["n_stages"] == 5 and kinds.count("rmsnorm_8bit") == 2 and kinds.count("rotary") == 1 and program.info["n_single_ops"] == 0
    ins, outs = [B.to_device(inputs[t.name], t.dtype) for t in spec.inputs], B.alloc_outputs(spec)
    ws = program.make_workspace()
    stream = torch.cuda.current_stream().cuda_stream
    address = [t.data_ptr() for t in ins], [t.data_ptr() for t in outs], ws.data_ptr(), ws.numel(), stream
    program.bind(*address)()
    torch.cuda.synchronize()
    whole = {n: B.to_host(t, d).copy() for (n, d), t in zip(spec.outputs, outs)}
    _check(spec, inputs, whole, dtype)
    for t in outs:
        t.view(torch.uint8).fill_(0x7F)
    for stage in range(program.info["n_stages"]):
        program.bind_stage(stage, *address)()
    torch.cuda.synchronize()
    for (n, d), t in zip(spec.outputs, outs):
        assert np.array_equal(B.to_host(t, d).view(np.uint8), whole[n].view(np.uint8)), n
