"""How the backward residual step shares rows out, as its workspace shows it: a slot of sums for each team."""
import pytest
import torch

from paper_2609_32197_b200 import binding

SMS = 148


def teams(dim, dtype, norm_y="none", weights=None, rows=1 << 20):
    step = binding.make_gated_norm(rows, dim, 0, norm_y, "layer", dtype=dtype, weight_dtype=weights)
    slots = (binding.sparsp_gated_norm_workspace_bytes(step) - 256) // (4 * dim)
    return (slots - 4 * 4 * SMS) // 10


@pytest.mark.parametrize("norm_y", ["none", "layer"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim", [2568, 2816, 3080, 3328, 3456, 3584, 3840, 4096, 4608, 5120])
def test_two_rows_at_a_time(dim, dtype, norm_y):
    """16 values a thread, of which a multiprocessor's registers hold 384: more teams would wait for others to end."""
    threads = -(-dim // 512) * 32
    for weights in (dtype, torch.float32):
        assert teams(dim, dtype, norm_y, weights) == SMS * max(1, 384 // threads)


@pytest.mark.parametrize("dim,dtype,ctas", [(512, torch.bfloat16, 2), (256, torch.bfloat16, 2), (512, torch.float32, 2),
                                            (128, torch.float32, 4)])
def test_rows_of_a_warp_with_a_norm_of_y(dim, dtype, ctas):
    lanes = min(32, dim // (8 if dtype != torch.float32 else 4))
    assert teams(dim, dtype, "rms") == SMS * ctas * (128 // lanes)
