"""4-bit operands and their product against the plain 64-bit form.

The quantisation is exact: codes, scales and values are those of the definition.  Bounds of the product: a sum of K
products in fp32, added 16 at a time, is off by at most (K / 16 + 8) 2^-23 of the sum of the products' magnitudes
(additions may cut instead of rounding); then one fp32 operation with the bias and one rounding."""
import pytest
import torch

import fp4_reference as ref
from layer_reference import F32, TINY, UNIT, close
from paper_2609_32197_b200 import binding

pytestmark = pytest.mark.gpu
BF, HF, F4 = torch.bfloat16, torch.float16, torch.float32


def matrix(rows, cols, dtype, seed=0, spread=2.0):
    """Values whose blocks have different sizes."""
    gen = torch.Generator().manual_seed(seed)
    size = torch.exp(spread * torch.randn(rows, cols // 16, generator=gen)).repeat_interleave(16, 1)
    return (torch.randn(rows, cols, generator=gen) * size).to(dtype).cuda()


def quantized(x, fmt, exponent=0, values=False):
    rows, cols = x.shape
    fp4 = binding.make_fp4(rows, cols, fmt, exponent, x.dtype, x.stride(0))
    codes, scales = binding.make_fp4_operand(fp4)
    codes.fill_(0xA5)
    scales.fill_(0xA5)
    out = torch.full_like(x, 7.0) if values else None
    if values and x.stride(0) != cols:
        out = torch.full((rows, x.stride(0)), 7.0, dtype=x.dtype, device="cuda")[:, :cols]
    binding.sparsp_fp4_quantize(fp4, x, codes, scales, out)
    return (codes, scales, out) if values else (codes, scales)


def check_quantized(x, fmt, exponent=0):
    codes, scales, values = quantized(x, fmt, exponent, True)
    want_scales, want_codes, want_values = ref.quantize(x, fmt, exponent)
    at, n = ref.scale_places(*x.shape, fmt)
    assert scales.numel() == n
    laid = torch.zeros(n, dtype=torch.uint8)
    laid[at] = want_scales.cpu()
    assert torch.equal(scales.cpu(), laid)
    bad = ~want_values.isfinite()
    got = ref.unpack_codes(codes)
    # (where a scale is NaN the codes mean nothing)
    assert torch.equal(torch.where(bad, 0, got.long()), torch.where(bad, 0, want_codes))
    want = want_values.to(x.dtype)
    assert torch.equal(values.isnan(), want.isnan())
    assert torch.equal(torch.nan_to_num(values), torch.nan_to_num(want))


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
@pytest.mark.parametrize("dtype", [BF, HF, F4])
@pytest.mark.parametrize("rows,cols", [(1, 32), (3, 96), (129, 160), (40, 1024), (7, 1056), (257, 2080), (1000, 320)])
def test_quantize(fmt, dtype, rows, cols):
    check_quantized(matrix(rows, cols, dtype, rows + cols, 2.0 if dtype != HF else 1.0), fmt)


@pytest.mark.parametrize("exponent", [-100, -14, -3, 5, 20, 100])
@pytest.mark.parametrize("dtype", [BF, F4])
def test_quantize_exponent(exponent, dtype):
    check_quantized((matrix(67, 192, F4, exponent + 200, 3.0) * 2.0 ** exponent).to(dtype), "nvfp4", exponent)


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
def test_quantize_borders(fmt):
    """Every border between two values, and one step of fp32 to either side, under scales of every mantissa."""
    b = ref.BLOCK[fmt]
    middles = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    row = torch.cat((torch.tensor([6.0]), middles, torch.nextafter(middles, torch.tensor(9.0)), torch.zeros(32))[:]) [:b]
    below = torch.cat((torch.tensor([-6.0]), torch.nextafter(middles, torch.tensor(0.0)), -middles, torch.zeros(32)))[:b]
    steps = torch.arange(8, 16).float() / 8 if fmt == "nvfp4" else torch.ones(1)
    blocks = [s * 2.0 ** e * r for s in steps for e in (-5, 0, 3) for r in (row, below)]
    x = torch.cat(blocks + [torch.zeros(-len(blocks) * b % 32)])[None].cuda()
    check_quantized(x, fmt)


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
@pytest.mark.parametrize("dtype", [BF, F4])
def test_quantize_extremes(fmt, dtype):
    """Zeros, the type's largest and smallest values, infinities and NaN, each in a block of its own beside others."""
    x = matrix(5, 256, dtype, 3, 0.5)
    most, least = torch.finfo(dtype).max, 2.0 ** -133 if dtype == BF else 2.0 ** -149
    x[0, :64] = 0
    x[1, 32:64] = most
    x[1, 65] = -most
    x[2, :32] = least
    x[2, 40] = 2.0 ** -126
    x[3, 5], x[3, 70], x[3, 130] = float("inf"), float("-inf"), float("nan")
    x[4, 100] = 2.0 ** -140 if dtype == F4 else -least
    check_quantized(x, fmt)


@pytest.mark.parametrize("dtype", [BF, F4])
@pytest.mark.parametrize("exponent,size", [(-100, 1e30), (-100, 3.0), (100, 1e-3), (100, 1e38), (-3, 3e38)])
def test_quantize_with_an_exponent_far_off(exponent, size, dtype):
    """Scales of 448 under values that do not fit, and of zero over values that are too small."""
    check_quantized((matrix(9, 96, F4, 77, 0.5) * size).clamp(-3.3e38, 3.3e38).to(dtype), "nvfp4", exponent)


def test_quantize_strided_and_in_place():
    wide = matrix(130, 512, BF, 5)
    x = wide[:, 64:416]
    check_quantized(x, "mxfp4")
    before, want = wide.clone(), ref.quantize(x, "mxfp4")[2].to(BF)
    fp4 = binding.make_fp4(130, 352, "mxfp4", 0, BF, 512)
    binding.sparsp_fp4_quantize(fp4, x, *binding.make_fp4_operand(fp4), x)
    assert torch.equal(x, want)
    before[:, 64:416] = want
    assert torch.equal(wide, before)  # nothing between the rows


def product(a, b, fmt, exponents, dtype, bias, stride_c=0):
    m, k = a.shape
    n = b.shape[0]
    qa, qb = quantized(a, fmt, exponents[0]), quantized(b, fmt, exponents[1])
    d = binding.make_fp4_product(m, n, k, fmt, sum(exponents), dtype, stride_c)
    ws = binding.make_fp4_product_workspace(d)
    c = torch.full((m, stride_c or n), 3.0, dtype=dtype, device="cuda")
    for _ in range(2):  # (the second call finds the workspace as the first left it)
        binding.sparsp_fp4_product(d, *qa, *qb, bias, c, ws)
    assert binding.sparsp_status(ws) == binding.SPARSP_OK
    return c


def check_product(m, n, k, fmt, dtype, with_bias=True, exponents=(0, 0), stride_c=0, in_type=BF, seed=0):
    a, b = matrix(m, k, in_type, seed + 1, 0.7), matrix(n, k, in_type, seed + 2, 0.7) * k ** -0.5
    a, b = a * 2.0 ** exponents[0], b * 2.0 ** exponents[1]
    bias = torch.randn(n, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda() if with_bias else None
    c = product(a, b, fmt, exponents, dtype, bias, stride_c)
    va, vb = ref.quantize(a, fmt, exponents[0])[2], ref.quantize(b, fmt, exponents[1])[2]
    want = va @ vb.T + (bias.double() if with_bias else 0.0)
    off = (k / 16 + 8) * 2.0 ** -23 * (va.abs() @ vb.abs().T) + F32 * want.abs()
    close(c[:, :n], want, off + UNIT[dtype] * (want.abs() + off) + TINY[dtype], "C")
    assert bool((c[:, n:] == 3.0).all())


SIZES = [(1, 8, 32), (1, 128, 256), (2, 136, 96), (5, 1000, 544), (16, 264, 2048), (33, 520, 288), (64, 4096, 512),
         (100, 256, 1056), (128, 384, 800), (129, 264, 64), (200, 248, 352), (226, 640, 480), (256, 256, 256),
         (257, 520, 1024), (1003, 1160, 1056), (513, 16, 320), (2100, 72, 192)]


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_product(fmt, m, n, k):
    check_product(m, n, k, fmt, BF, with_bias=(m + n) % 16 < 8)


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
@pytest.mark.parametrize("dtype", [HF, F4])
@pytest.mark.parametrize("m,n,k", [(1, 264, 544), (70, 136, 288), (300, 392, 416)])
def test_product_types(fmt, dtype, m, n, k):
    check_product(m, n, k, fmt, dtype, in_type=dtype)
    check_product(m, n, k, fmt, dtype, False, stride_c=n + 24)


@pytest.mark.parametrize("m", [3, 300])
def test_product_exponents(m):
    check_product(m, 264, 320, "nvfp4", BF, exponents=(3, -14))
    check_product(m, 264, 320, "nvfp4", F4, exponents=(-30, 40))


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
@pytest.mark.parametrize("m", [4, 300])
def test_product_nan_stays_in_its_row_and_column(fmt, m):
    a, b = matrix(m, 608, BF, 1, 0.5), matrix(264, 608, BF, 2, 0.5)
    a[m - 2, 600], b[7, 3], b[200, 400] = float("nan"), float("inf"), float("-inf")
    c = product(a, b, fmt, (0, 0), F4, None)
    want = torch.zeros(m, 264, dtype=torch.bool, device="cuda")
    want[m - 2], want[:, 7], want[:, 200] = True, True, True
    assert torch.equal(c.isnan(), want) and not bool(c.isinf().any())


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
@pytest.mark.parametrize("m,n,k", [(1, 512, 4096), (77, 1000, 2080), (1500, 2100 // 8 * 8, 1056)])
def test_same_bits(fmt, m, n, k):
    a, b = matrix(m, k, BF, 4, 0.7), matrix(n, k, BF, 5, 0.7)
    first = product(a, b, fmt, (0, 0), F4, None)
    for _ in range(3):
        assert torch.equal(product(a, b, fmt, (0, 0), F4, None), first)


def test_many_tiles_and_rounds():
    """More tiles than pairs of multiprocessors, several each, and a ragged last one in both directions."""
    check_product(256 * 13 + 5, 256 * 19 + 8, 288, "nvfp4", BF)
    check_product(256 * 40 + 100, 1032, 768, "mxfp4", BF)


def test_no_rows():
    for fmt in ("mxfp4", "nvfp4"):
        d = binding.make_fp4_product(0, 8, 32, fmt)
        ws = binding.make_fp4_product_workspace(d)
        binding.sparsp_fp4_product(d, None, None, None, None, None, None, ws)
        fp4 = binding.make_fp4(0, 32, fmt)
        binding.sparsp_fp4_quantize(fp4, None, None, None, None)
