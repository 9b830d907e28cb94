"""Host side of the 4-bit operands: sizes, and what the calls refuse before anything is launched."""
import pytest
import torch

from paper_2609_32197_b200 import binding
from test_layer_host import At, INVALID, UNSUPPORTED, no_stream, refused  # noqa: F401


@pytest.mark.parametrize("rows,cols,fmt,groups", [(1, 32, "mxfp4", 1), (128, 128, "mxfp4", 1), (129, 160, "mxfp4", 4),
                                                  (1, 32, "nvfp4", 1), (128, 64, "nvfp4", 1), (300, 96, "nvfp4", 6)])
def test_scales_bytes(rows, cols, fmt, groups):
    assert binding.sparsp_fp4_scales_bytes(binding.make_fp4(rows, cols, fmt)) == 512 * groups
    assert binding.sparsp_fp4_scales_bytes(binding.make_fp4(0, cols, fmt)) == 0


@pytest.mark.parametrize("code,change", [
    (INVALID, {"format": 2}), (INVALID, {"format": -1}), (INVALID, {"exponent": 1}), (INVALID, {"format": 1, "exponent": 101}),
    (INVALID, {"format": 1, "exponent": -101}), (INVALID, {"rows": -1}), (INVALID, {"cols": 0}), (UNSUPPORTED, {"cols": 48}),
    (UNSUPPORTED, {"cols": (1 << 28) + 32, "stride_x": 1 << 30}), (INVALID, {"stride_x": 56}), (INVALID, {"stride_x": 68}),
    (INVALID, {"dtype": 3}), (UNSUPPORTED, {"rows": 1 << 31})])
def test_refused_operands(code, change):
    fp4 = binding.make_fp4(4, 64)
    for k, v in change.items():
        setattr(fp4, k, v)
    refused(code, binding.sparsp_fp4_scales_bytes, fp4)
    refused(code, binding.sparsp_fp4_quantize, fp4, At(), At(8192), At(16384), None)


def test_refused_operand_pointers():
    fp4 = binding.make_fp4(4, 64)
    good = [At(), At(8192), At(16384), At(1 << 20)]
    for i in range(4):
        refused(INVALID, binding.sparsp_fp4_quantize, fp4, *(At(1032) if i == j else g for j, g in enumerate(good)))
        if i < 3:
            refused(INVALID, binding.sparsp_fp4_quantize, fp4, *(None if i == j else g for j, g in enumerate(good)))
    for i, j in ((1, 0), (2, 0), (1, 2), (1, 3), (2, 3)):  # codes and scales apart from everything
        args = list(good)
        args[i] = args[j]
        refused(INVALID, binding.sparsp_fp4_quantize, fp4, *args)
    with pytest.raises(KeyError):
        binding.make_fp4(4, 64, "fp4")
    with pytest.raises(ValueError):
        binding.make_fp4(4, 64, dtype=torch.float64)


@pytest.mark.parametrize("code,change", [
    (INVALID, {"format": 2}), (INVALID, {"exponent": 2}), (INVALID, {"format": 1, "exponent": 127}), (INVALID, {"rows": -1}),
    (INVALID, {"cols": 0}), (INVALID, {"depth": 0}), (UNSUPPORTED, {"cols": 12}), (UNSUPPORTED, {"depth": 80}),
    (INVALID, {"stride_c": 8}), (INVALID, {"stride_c": 36}), (UNSUPPORTED, {"stride_c": (1 << 37) + 8}), (INVALID, {"dtype": -1}),
    (UNSUPPORTED, {"rows": 1 << 31}), (UNSUPPORTED, {"depth": (1 << 28) + 32}),
    (UNSUPPORTED, {"cols": (1 << 28) + 8, "stride_c": 1 << 30})])
def test_refused_products(code, change):
    d = binding.make_fp4_product(4, 32, 64)
    for k, v in change.items():
        setattr(d, k, v)
    refused(code, binding.sparsp_fp4_product_workspace_bytes, d)
    refused(code, binding.sparsp_fp4_product, d, At(), At(), At(), At(), None, At(1 << 20), At(1 << 21))


def test_refused_product_pointers():
    d = binding.make_fp4_product(4, 32, 64)
    good = [At(), At(8192), At(16384), At(32768), At(65536), At(1 << 20), At(1 << 21)]
    for i in range(7):
        refused(INVALID, binding.sparsp_fp4_product, d, *(At(1032) if i == j else g for j, g in enumerate(good)))
        if i != 4:
            refused(INVALID, binding.sparsp_fp4_product, d, *(None if i == j else g for j, g in enumerate(good)))
        if i < 5:
            refused(INVALID, binding.sparsp_fp4_product, d, *(good[i] if j == 5 else g for j, g in enumerate(good)))


def test_workspace_of_more_rows_serves_fewer():
    for fmt in ("mxfp4", "nvfp4"):
        for n, k in ((8, 32), (1160, 1056), (7680, 1920), (30720, 5120)):
            size = [binding.sparsp_fp4_product_workspace_bytes(binding.make_fp4_product(m, n, k, fmt))
                    for m in (0, 1, 16, 127, 128, 129, 256, 1000, 5000, 75600)]
            assert size == sorted(size) and size[0] >= 256
