"""Group normalisation of float tensors whose outputs share memory runs op by op, in the host core under AddressSanitizer +
UndefinedBehaviorSanitizer (CPU only)."""
import os
import subprocess
import sys

import pytest

from .test_host_sanitizers import ROOT, _asan_runtime


def test_shared_outputs_run_op_by_op_where_the_workspace_is_large_enough():
    runtime = _asan_runtime()
    if runtime is None:
        pytest.skip("the host compiler's AddressSanitizer runtime is not installed")
    from paper_2009_10924_amd.build import build_host_sanitized
    env = dict(os.environ, FUSION_STITCHING_LIB=build_host_sanitized(), LD_PRELOAD=runtime, FS_CODEGEN_CACHE_DIR="",
               ASAN_OPTIONS="detect_leaks=0:abort_on_error=1:halt_on_error=1", UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    env.pop("FS_STUB_COMPILE_OK", None)
    r = subprocess.run([sys.executable, os.path.join(ROOT, "tests", "host_sanitizer_shared_outputs.py")], env=env, capture_output=True, text=True, timeout=900)
    tail = (r.stdout + r.stderr)[-4000:]
    assert r.returncode == 0, tail
    assert "no report" in r.stdout and "ERROR: AddressSanitizer" not in r.stderr and "runtime error:" not in r.stderr, tail
