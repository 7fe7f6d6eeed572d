"""Run as a child process by tests/test_shared_outputs.py, with the sanitizer build of the host core: what calls whose outputs share
memory launch.  Launches are checked and counted by the host stub; nothing runs."""
import ctypes
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

from paper_2009_10924_amd import binding as B                                            # noqa: E402
from workloads import (checkpoint_graph, group_norm_backward_graph, group_norm_graph)    # noqa: E402

WS = 1 << 46


def apart(n, base):
    return [base + (i << 40) for i in range(n)]


def refused(call, text):
    try:
        call()
    except B.FsError as e:
        assert e.code == -1 and "shares memory" in str(e) and text in str(e), e
        return
    raise AssertionError("not refused")


def launches(lib, call):
    before = lib.fs_stub_launch_count()
    call()
    return lib.fs_stub_launch_count() - before


def main():
    lib = B.load()
    lib.fs_stub_launch_count.restype = ctypes.c_long
    assert "host_san" in B.lib_path()
    for dtype in ("f32", "bf16"):
        for shape in ((2, 64, 4, 16), (1, 9000, 3, 5), (1, 60000, 32, 8), (3, 197, 5, 7)):
            for spec, out, over in ((group_norm_graph(*shape, dtype=dtype, act="none", keep="none"), 0, 0),
                                    (group_norm_graph(*shape, dtype=dtype, act="silu", keep="stats"), 0, 0),
                                    (group_norm_backward_graph(*shape, dtype=dtype, act="gelu", keep="stats"), 0, 2)):
                graph = B.Graph.from_spec(spec)
                plan, ops = B.Plan(graph), B.Plan(graph, "unfused")
                assert plan.info["pattern"].startswith("group_norm")
                need, need_ops = plan.info["workspace_bytes"], ops.info["workspace_bytes"]
                ins, outs = apart(len(spec.inputs), 1 << 44), apart(len(spec.outputs), 1 << 45)
                shared = list(outs)
                shared[out] = ins[over]
                assert need_ops > need
                # with the memory that the per-op plan takes: its launches; with less: refused, with the size; apart: the family's
                assert launches(lib, lambda: plan.execute_ptrs(ins, shared, WS, need_ops, 0)) == ops.info["n_kernels"] > plan.info["n_kernels"]
                assert launches(lib, lambda: plan.execute_ptrs(ins, outs, WS, need_ops, 0)) == plan.info["n_kernels"]
                refused(lambda: plan.execute_ptrs(ins, shared, WS, need_ops - 1, 0), f"{need_ops} bytes")
                refused(lambda: plan.execute_static_ptrs(ins, shared, 0), "shares memory")
                if need == 0:
                    refused(lambda: plan.execute_ptrs(ins, shared, 0, need_ops, 0), f"{need_ops} bytes")
                    refused(lambda: plan.execute_ptrs(ins, shared, WS + 8, need_ops, 0), f"{need_ops} bytes")
                # the same in a program: behind its own workspace
                prog = B.Program(graph)
                assert "pattern=group_norm" in prog.describe()
                own = (prog.info["workspace_bytes"] + 255) // 256 * 256
                assert launches(lib, prog.bind(ins, shared, WS, own + need_ops, 0)) == ops.info["n_kernels"]
                assert launches(lib, prog.bind(ins, outs, WS, own + need_ops, 0)) == plan.info["n_kernels"]
                refused(prog.bind(ins, shared, WS, own + need_ops - 1, 0), f"{need_ops} bytes")
        # graphs with 8-bit tensors came with the rule
        for spec in (group_norm_graph(2, 64, 4, 16, dtype, "silu", "checkpoint"), checkpoint_graph(8, 2, 64, dtype)):
            plan = B.Plan(B.Graph.from_spec(spec))
            ins, outs = apart(len(spec.inputs), 1 << 44), apart(len(spec.outputs), 1 << 45)
            refused(lambda: plan.execute_ptrs(ins, [ins[0]] + outs[1:], WS, 1 << 40, 0), "")
    print("shared outputs driver: no report")


if __name__ == "__main__":
    main()
