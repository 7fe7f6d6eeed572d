"""Run as a child process by tests/test_host_sanitizer_decoder.py, like host_sanitizer_checkpoints.py: dropout, 8-bit norms and rotary positions
through the sanitizer build of the host core, every candidate of graphs of one value up to the limit of 2^31 elements, the per-op plans and
a program of all of them.  Launches are checked and counted by the host stub; nothing runs."""
import ctypes
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

from paper_2009_10924_amd import binding as B                                            # noqa: E402
from workloads import (decoder_block_graph, dropout_backward_graph, dropout_graph, rmsnorm_8bit_graph,   # noqa: E402
                       rmsnorm_residual_backward_graph, rotary_graph)

MOST = (1 << 31) - 1
TYPES = ("f32", "f16", "bf16")


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
    for scheme, opts in [("auto", {}), ("unfused", {})] + [("auto", {"candidate": i}) for i in range(B.Plan(graph).info["n_candidates"])]:
        plan = B.Plan(graph, scheme, **opts)
        need = plan.info["workspace_bytes"]
        plan.execute_ptrs(ins, outs, 1 << 46, need, 0)
        if need <= B.FS_STATIC_SCRATCH_BYTES:
            plan.execute_static_ptrs(ins, outs, 0)
        plan.describe()
        plan.source()
        if plan.info["pattern"] == "rmsnorm_8bit":   # (a rotary op by itself turns in place, op by op)
            refused(lambda: plan.execute_ptrs(ins, [ins[0]] + outs[1:], 1 << 46, need, 0))
        if plan.info["pattern"] == "dropout":
            plan.execute_ptrs(ins, [ins[0]], 1 << 46, need, 0)
        if need:
            refused(lambda: plan.execute_ptrs(ins, outs, 1 << 46, need - 1, 0))
        refused(lambda: plan.execute_ptrs([ins[0] + 8] + ins[1:], outs, 1 << 46, need, 0))


def main():
    lib = B.load()
    lib.fs_stub_launch_count.restype = ctypes.c_long
    assert "host_san" in B.lib_path()
    for k, (rows, cols) in enumerate([(1, 1), (1, 8), (3, 7), (65, 131), (1000, 4096), (4097, 653), (2, 40001), (MOST, 1), (1, MOST), (3, MOST // 3), (MOST // 9, 9)]):
        dtype = TYPES[k % 3]
        run(dropout_graph(rows, cols, 0.1, dtype=dtype, act=("none", "gelu", "silu")[k % 3], bias=k % 2 == 0, residual=k % 2 == 1))
        run(dropout_backward_graph(rows, cols, 0.1, dtype=dtype, act="gelu", bias=k % 2 == 0, dbias=False))
        for p, bias, keep in ((0.0, False, "none"), (0.25, True, "stats")):
            run(rmsnorm_8bit_graph(rows, cols, dtype=dtype, p=p, bias=bias, keep=keep, normed=bias, rounded=bias))
        run(rmsnorm_8bit_graph(rows, cols, dtype=dtype, residual=False))
        if rows * cols < 1 << 26:
            run(dropout_backward_graph(rows, cols, 0.1, dtype=dtype, act="silu", bias=True, dbias=True))
            run(rmsnorm_residual_backward_graph(rows, cols, dtype=dtype, p=0.1))
    for k, (batch, seq, heads, dim, sections) in enumerate([(1, 1, (1,), 2, (1,)), (2, 33, (8, 2), 128, (16, 24, 24)), (3, 5, (5, 5), 80, (14, 15)), (1, 7, (3,), 25, (5, 2, 1, 3)),
                                                            (1, MOST // 2, (1,), 2, (1,)), (MOST // 2, 1, (1,), 2, (1,)), (1, 1, (MOST // 2,), 2, (1,)), (1, 1, (1,), MOST, (4096,)),
                                                            (9, 100, (64, 8), 8200, (4096,)), (2, 16384, (32, 8), 128, (64,))]):
        for inverse in (False, True):
            run(rotary_graph(batch, seq, heads, dim, sections, dtype=TYPES[k % 3], interleaved=k % 2 == 1, restart=k % 3 == 0, inverse=inverse, split=k % 2 == 0))
    program = B.Program(B.Graph.from_spec(decoder_block_graph()))
    program.describe()
    print(f"{lib.fs_stub_launch_count()} launches checked, no report")


if __name__ == "__main__":
    main()
