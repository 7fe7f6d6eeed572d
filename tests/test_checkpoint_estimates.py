"""What a plan says a checkpoint of long blocks will take, beside times measured on an MI355X (three sets of buffers in turn): a
workgroup per block, so few long blocks take as long as one does, whatever the memory could do."""
import pytest

from paper_2009_10924_amd import binding as B
from workloads import checkpoint_graph

# dtype, act, bias, (rows, block), us
MEASURED = [("bf16", "none", False, (1, 1 << 26), 7677.0), ("bf16", "none", False, (1, 1 << 22), 390.0), ("bf16", "gelu", True, (1, 1 << 22), 950.0),
            ("f32", "none", False, (1, 1 << 22), 511.0), ("f32", "silu", True, (1, 1 << 20), 218.0), ("bf16", "gelu", False, (16, 1 << 20), 182.0),
            ("f32", "gelu", False, (16, 1 << 18), 43.2), ("bf16", "none", False, (3, 40000), 4.34), ("f16", "silu", True, (64, 100000), 22.8),
            ("f32", "none", False, (200, 40000), 10.6), ("bf16", "gelu", True, (256, 70000), 22.3), ("bf16", "none", False, (700, 70000), 37.7),
            ("f32", "gelu", True, (1000, 33001), 75.1), ("bf16", "silu", False, (2000, 33000), 72.8), ("bf16", "none", False, (5, 33001), 6.38),
            ("f32", "none", False, (1, 17000), 3.62), ("f32", "silu", False, (4, 33333), 6.29)]


@pytest.mark.parametrize("dtype,act,bias,shape,us", MEASURED)
def test_long_blocks(dtype, act, bias, shape, us):
    info = B.Plan(B.Graph.from_spec(checkpoint_graph(shape[0], 1, shape[1], dtype, act, bias))).info
    assert info["kernel"].startswith("checkpoint_long")
    assert us / 1.5 <= info["predicted_us"] <= us * 1.5, (us, info["predicted_us"])
