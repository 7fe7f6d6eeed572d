"""Vectors at any element of a tensor: every load and store of them says the alignment that it can count on, that of one element."""
import os
import shutil
import subprocess

import pytest

from paper_2009_10924_amd.build import CSRC, HIPCC

SOURCE = """
#include <hip/hip_runtime.h>
#include "vec_access.hpp"
namespace fsk {
template <typename T, int VEC>
__device__ void copy(const T* from, T* to, bool stream) {
  float v[VEC];
  VecIo<T, VEC>::widen(VecIo<T, VEC>::template load<false>(from), v);
  store_as<VecIo<T, VEC>>(stream, to, v);
  VecIo<T, VEC>::widen(VecIo<T, VEC>::template load<true>(from), v);
  VecIo<T, VEC>::store(to, v);
}
__global__ void all(const float* f, const f16_t* h, const bf16_t* b, const e4m3_t* q, float* F, f16_t* H, bf16_t* B, e4m3_t* Q, bool stream) {
  copy<float, 4>(f, F, stream), copy<f16_t, 8>(h, H, stream), copy<bf16_t, 8>(b, B, stream), copy<e4m3_t, 8>(q, Q, stream), copy<e4m3_t, 4>(q, Q, stream);
  copy<float, 1>(f, F, stream), copy<f16_t, 1>(h, H, stream), copy<bf16_t, 1>(b, B, stream), copy<e4m3_t, 1>(q, Q, stream);
}
}
"""


def test_no_access_claims_more_than_an_elements_alignment(tmp_path):
    if not (shutil.which(HIPCC) or os.path.exists(HIPCC)):
        pytest.skip("no hipcc")
    path = tmp_path / "accesses.hip"
    path.write_text(SOURCE)
    asm = tmp_path / "accesses.ll"
    r = subprocess.run([HIPCC, "-O1", "-std=c++17", "--offload-arch=gfx950", "-Werror=align-mismatch", f"-I{CSRC}/kernels", "--cuda-device-only", "-S",
                        "-emit-llvm", "-o", str(asm), str(path)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    accesses = [line for line in asm.read_text().splitlines() if " addrspace(1)" in line and (" load <" in line or "store <" in line)]
    assert len(accesses) >= 8, accesses   # four vector types, a load and a store of each at least
    for line in accesses:
        assert int(line.split("align ")[1].split(",")[0]) <= 4, line
