"""Zeros of either sign, and negative values that are lost below fp32's range, keep their sign in the codes."""
import pytest
import torch

from test_gpu_fp4 import BF, F4, HF, check_quantized, matrix

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
@pytest.mark.parametrize("dtype", [BF, HF, F4])
def test_negative_zeros(fmt, dtype):
    x = matrix(5, 96, dtype, 1, 0.5)
    x[0, ::3] = -0.0
    x[1, 1::2] = 0.0
    x[2, 32:64] = -0.0  # blocks of nothing else
    x[3] = -0.0
    x[4, :48] = torch.where(torch.arange(48, device="cuda") % 2 == 0, -0.0, 0.0).to(dtype)
    check_quantized(x, fmt)


@pytest.mark.parametrize("dtype", [BF, F4])
def test_negative_values_that_are_lost(dtype):
    """Under an exponent of 100 they leave fp32's range on their way to the scale; beside values that keep the scale above zero,
    and alone, where it is zero."""
    x = matrix(4, 64, F4, 2, 0.5).abs() * 2.0 ** 100
    x[0, ::2], x[1, 5] = -(2.0 ** -60), -(2.0 ** -126)
    x[2] = -(2.0 ** -100)
    x[3, :16] = -0.0
    check_quantized(x.to(dtype), "nvfp4", 100)


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
@pytest.mark.parametrize("dtype", [BF, HF, F4])
def test_negative_values_that_round_to_zero(fmt, dtype):
    x = matrix(3, 64, dtype, 3, 0.1)
    x[:, ::4], x[:, 0] = -2.0 ** -12, 6.0
    check_quantized(x, fmt)
