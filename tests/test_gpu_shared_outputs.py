"""Group normalisation of float tensors in place: a call whose outputs share memory gives what its ops give one by one."""
import numpy as np
import pytest

from oracle import oracle as O
from paper_2009_10924_amd import binding as B
from workloads import group_norm_backward_graph, group_norm_graph, make_inputs

from .test_gpu_checkpoint import within
from .test_gpu_group_norm import backward_bounds, forward_bounds

pytestmark = pytest.mark.gpu

# (forward / backward, act, keep, the input that the first output takes the place of): one that no op reads any more when it is written
CASES = [("forward", "silu", "stats", "x"), ("forward", "none", "none", "x"), ("backward", "gelu", "stats", "dy"), ("backward", "silu", "stats", "x")]
SHAPES = [(2, 64, 4, 16), (3, 197, 5, 7), (1, 9000, 3, 5), (1, 60000, 32, 8)]


def ready(direction, act, keep, over, shape, dtype):
    spec = (group_norm_graph if direction == "forward" else group_norm_backward_graph)(*shape, dtype=dtype, act=act, keep=keep)
    inp = make_inputs(spec, seed=3)
    env = O.evaluate(spec, inp, keep_all=True)
    names = [t.name for t in spec.inputs]
    dev = [B.to_device(inp[t.name], t.dtype) for t in spec.inputs]
    outs = B.alloc_outputs(spec)
    outs[0] = dev[names.index(over)]
    allowed = forward_bounds(spec, env, act, dtype) if direction == "forward" else backward_bounds(env, dtype)
    kept = dev[names.index(over)].clone()

    def check(what):
        for (name, d), t in zip(spec.outputs, outs):
            within(O.to_f64(B.to_host(t, d), d).reshape(env[name].shape), env[name], allowed[name], f"{spec.name} {what} {name}")
        outs[0].copy_(kept)
        for t in outs[1:]:
            t.fill_(float("nan"))
    return spec, dev, outs, check


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(c))
def test_first_output_in_the_place_of_an_input(case, shape, dtype):
    import torch
    spec, dev, outs, check = ready(*case, shape, dtype)
    graph = B.Graph.from_spec(spec)
    plan, prog = B.Plan(graph), B.Program(graph)
    need = B.Plan(graph, "unfused").info["workspace_bytes"]
    ins_p, outs_p = [t.data_ptr() for t in dev], [t.data_ptr() for t in outs]
    stream = torch.cuda.current_stream().cuda_stream
    own = (prog.info["workspace_bytes"] + 255) // 256 * 256
    ws = torch.empty(own + need, dtype=torch.uint8, device="cuda")
    with pytest.raises(B.FsError, match="shares memory"):
        plan.execute_ptrs(ins_p, outs_p, ws.data_ptr(), need - 1, stream)
    for what, call in (("plan", lambda: plan.execute_ptrs(ins_p, outs_p, ws.data_ptr(), need, stream)),
                       ("program", prog.bind(ins_p, outs_p, ws.data_ptr(), own + need, stream))):
        ws.fill_(0xFF)
        call()
        torch.cuda.synchronize()
        check(what)


def test_in_place_replayed_from_a_graph():
    import torch
    spec, dev, outs, check = ready("forward", "silu", "stats", "x", (2, 64, 4, 16), "f32")
    graph = B.Graph.from_spec(spec)
    plan, need = B.Plan(graph), B.Plan(graph, "unfused").info["workspace_bytes"]
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    captured = torch.cuda.CUDAGraph()
    with torch.cuda.graph(captured, stream=side):
        plan.execute_ptrs([t.data_ptr() for t in dev], [t.data_ptr() for t in outs], ws.data_ptr(), need, torch.cuda.current_stream().cuda_stream)
    for replay in range(3):
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        captured.replay()
        torch.cuda.synchronize()
        check(f"replay {replay}")
