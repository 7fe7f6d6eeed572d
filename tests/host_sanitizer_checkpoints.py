"""Run as a child process by tests/test_host_sanitizer_checkpoints.py, like host_sanitizer_driver.py: group normalisation and 8-bit
checkpoints through the sanitizer build of the host core, every candidate of graphs of one value up to the limit of 2^31 elements, the
per-op plans, a program of all four, and the refusals.  Launches are checked and counted by the host stub; nothing runs."""
import ctypes
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

from paper_2009_10924_amd import binding as B                                            # noqa: E402
from workloads import (checkpoint_backward_graph, checkpoint_graph, checkpointed_block_graph, group_norm_backward_graph,  # noqa: E402
                       group_norm_graph)

MOST = (1 << 31) - 1


def apart(n, base):
    return [base + (i << 40) for i in range(n)]


def refused(call):
    try:
        call()
    except B.FsError as e:
        assert e.code in (-1, -2, -3, -4, -5, -6, -7, -8), e
        return
    raise AssertionError("not refused")


def run(spec):
    graph = B.Graph.from_spec(spec)
    ins, outs = apart(len(spec.inputs), 1 << 44), apart(len(spec.outputs), 1 << 45)
    for opts in [("auto", {}), ("unfused", {})] + [("auto", {"candidate": i}) for i in range(B.Plan(graph).info["n_candidates"])]:
        plan = B.Plan(graph, opts[0], **opts[1])
        need = plan.info["workspace_bytes"]
        plan.execute_ptrs(ins, outs, 1 << 46, need, 0)
        if need <= B.FS_STATIC_SCRATCH_BYTES:
            plan.execute_static_ptrs(ins, outs, 0)
        plan.describe()
        plan.source()
        if plan.info["pattern"] != "unfused":
            refused(lambda: plan.execute_ptrs(ins, [ins[0]] + outs[1:], 1 << 46, need, 0))
        if need:
            refused(lambda: plan.execute_ptrs(ins, outs, 1 << 46, need - 1, 0))
            refused(lambda: plan.execute_ptrs(ins, outs, 0, need, 0))
        refused(lambda: plan.execute_ptrs([ins[0] + 8] + ins[1:], outs, 1 << 46, need, 0))


def main():
    lib = B.load()
    lib.fs_stub_launch_count.restype = ctypes.c_long
    assert "host_san" in B.lib_path()
    for k, shape in enumerate([(1, 1, 1, 1), (3, 197, 5, 7), (2, 33, 32, 10), (2, 9000, 4, 10), (1, 60000, 32, 8), (1, 5, 1, 2500), (20000, 1, 2, 4), (MOST, 1, 1, 1),
                               (1, MOST, 1, 1), (1, 1, MOST, 1), (1, 1, 1, MOST), (MOST // 64, 1, 64, 1), (2, 1 << 20, 32, 31), (70000, 1024, 4, 4)]):
        for act, keep in (("none", "none"), ("silu", "stats"), ("gelu", "checkpoint")):
            run(group_norm_graph(*shape, dtype=("f32", "f16", "bf16")[k % 3], act=act, keep=keep))
            if keep != "none":
                run(group_norm_backward_graph(*shape, dtype=("f32", "f16", "bf16")[k % 3], act=act, keep=keep))
    for k, shape in enumerate([(1, 1, 1), (7, 3, 100), (64, 4, 32), (5, 1, 1537), (3, 1, 70001), (MOST, 1, 1), (1, MOST, 1), (1, 1, MOST), (MOST // 7, 1, 7), (2000000, 16, 64)]):
        for act, more in (("none", False), ("gelu", True), ("silu", False), ("silu", True)):
            run(checkpoint_graph(*shape, dtype=("f32", "f16", "bf16")[k % 3], act=act, bias=more))
            run(checkpoint_backward_graph(*shape, dtype=("f32", "f16", "bf16")[k % 3], act=act, dbias=more))
    for sizes in ((2, 64, 4, 16, 256, 64), (1, 1, 1, 1, 1, 1), (3, 50, 5, 7, 100, 50)):
        spec = checkpointed_block_graph(*sizes)
        for opts in ({}, {"no_joint_folds": True}, {"no_packing": True, "no_remote_fusion": True}, {"top_k": 1, "beam_width": 1}):
            prog = B.Program(B.Graph.from_spec(spec), **opts)
            ws, ins, outs = prog.info["workspace_bytes"], apart(len(spec.inputs), 1 << 44), apart(len(spec.outputs), 1 << 45)
            prog.bind(ins, outs, 1 << 46, ws, 0)()
            for stage in range(prog.info["n_stages"]):
                prog.bind_stage(stage, ins, outs, 1 << 46, ws, 0)()
            prog.describe()
            prog.patterns()
            refused(prog.bind(ins, outs[:-1] + outs[-2:-1], 1 << 46, ws, 0))
    launches = lib.fs_stub_launch_count()
    assert launches > 1000, launches
    print(f"host sanitizer driver: {launches} checked launches, no report")


if __name__ == "__main__":
    main()
