"""Products of the longest rows that are allowed: a tile's products alone take longer than any other wait of the kernel may."""
import pytest
import torch

from paper_2609_32197_b200 import binding

pytestmark = pytest.mark.gpu


def operand(rows, depth):
    """Ones at both ends of each row, all scales 1."""
    codes = torch.zeros(rows, depth // 2, dtype=torch.uint8, device="cuda")
    codes[:, :32] = codes[:, -16:] = 0x22
    scales = torch.full((binding.sparsp_fp4_scales_bytes(binding.make_fp4(rows, depth)),), 127, dtype=torch.uint8, device="cuda")
    return codes, scales


@pytest.mark.parametrize("rows", [1, 129])
def test_rows_of_268_million_values(rows):
    cols, depth = 8, 1 << 28
    a, b = operand(rows, depth), operand(cols, depth)
    a[0][rows - 1, depth // 4] = b[0][cols - 1, depth // 4] = 0x07  # 6 times 6, once
    d = binding.make_fp4_product(rows, cols, depth, dtype=torch.float32)
    ws = binding.make_fp4_product_workspace(d)
    c = torch.full((rows, cols), float("nan"), device="cuda")
    binding.sparsp_fp4_product(d, *a, *b, None, c, ws)
    assert binding.sparsp_status(ws) == binding.SPARSP_OK
    want = torch.full((rows, cols), 96.0, device="cuda")
    want[rows - 1, cols - 1] += 36.0
    assert torch.equal(c, want)
