"""Layer norm against the plain 64-bit form.

Bounds, with u = 2^-24 and D values a row: a sum of D terms over a tree of depth log2 D after at most 32 terms a thread is
off by at most 48 u of the sum of its terms' magnitudes.  So mean is within 50 u max|x| and the deviations x - mean within
52 u max|x|; rstd is within (104 u max|x| rstd + 60 u) of itself; y is then within
|w| rstd 52 u max|x| + |xh w| (104 u max|x| rstd + 70 u) + the rounding of the stored value."""
import pytest
import torch

from layer_reference import F32, TINY, UNIT, close, layer_norm, layer_norm_back
from paper_2609_32197_b200 import binding

pytestmark = pytest.mark.gpu
EPS = 1e-5
BF, HF, FL = torch.bfloat16, torch.float16, torch.float32


def inputs(rows, dim, groups, dtype, wtype, offset=0.5, seed=0):
    gen = torch.Generator().manual_seed(seed)
    x = (torch.randn(rows, dim, generator=gen) * (1 + 3 * torch.rand(dim, generator=gen)) + offset).to(dtype).cuda()
    w = (1 + 0.3 * torch.randn(groups, dim, generator=gen)).to(wtype).cuda()
    b = (0.3 * torch.randn(groups, dim, generator=gen)).to(wtype).cuda()
    dy = torch.randn(rows, dim, generator=gen).to(dtype).cuda()
    return x, w, b, dy


def fwd_bounds(x, w, want, mean, rstd, per, dtype):
    top = x.abs().amax(1).clamp(min=1e-30)
    off_mean = 50 * F32 * top
    off_rstd = rstd * (104 * F32 * top * rstd + 60 * F32)
    g = torch.arange(x.shape[0], device=x.device) // per
    wa = torch.ones_like(x) if w is None else w[g].abs()
    xh = ((x - mean[:, None]) * rstd[:, None]).abs()
    off_y = wa * (rstd * 52 * F32 * top)[:, None] + xh * wa * (104 * F32 * top * rstd + 70 * F32)[:, None]
    return off_y + UNIT[dtype] * (want.abs() + off_y) + 4 * F32 * want.abs() + TINY[dtype], off_mean, off_rstd


SHAPES = [
    # rows, dim, groups, dtype, weights
    (1, 1, 1, BF, BF), (1, 8, 1, BF, FL), (3, 64, 1, HF, HF), (65, 128, 1, BF, BF), (33, 257, 1, BF, BF),
    (40, 512, 4, BF, FL), (12, 520, 3, HF, FL), (7, 1000, 1, FL, FL), (9, 1921, 3, FL, FL), (5, 2049, 1, HF, HF),
    (11, 4096, 1, BF, BF), (3, 5120, 3, BF, FL), (4, 8192, 1, FL, FL), (3, 8200, 1, BF, BF), (2, 12289, 1, BF, FL),
    (2, 16384, 1, FL, FL), (2, 16383, 1, FL, FL), (2, 16384, 2, BF, BF), (1500, 96, 1, BF, BF), (6000, 24, 5, FL, FL),
    (700, 640, 7, BF, BF), (1301, 1032, 1, BF, BF), (5000, 3, 5000, FL, FL), (9000, 136, 9, HF, FL),
]


@pytest.mark.parametrize("rows,dim,groups,dtype,wtype", SHAPES)
def test_forward(rows, dim, groups, dtype, wtype):
    per = -(-rows // groups)
    x, w, b, _ = inputs(rows, dim, groups, dtype, wtype)
    norm = binding.make_norm(rows, dim, per, EPS, dtype, wtype)
    y = torch.full_like(x, float("nan"))
    mean, rstd = (torch.full((rows,), float("nan"), device="cuda") for _ in range(2))
    binding.sparsp_layer_norm_fwd(norm, x, w, b, y, mean, rstd)
    want, m, r = layer_norm(x.double(), w.double(), b.double(), EPS, per)
    by, bm, br = fwd_bounds(x.double(), w.double(), want, m, r, per, dtype)
    close(mean, m, bm, "mean")
    close(rstd, r, br, "rstd")
    close(y, want, by, "y")
    again = x.clone()  # in place, without statistics
    binding.sparsp_layer_norm_fwd(norm, again, w, b, again, None, None)
    assert torch.equal(again, y)


@pytest.mark.parametrize("rows,dim,groups,dtype,wtype", SHAPES)
def test_backward(rows, dim, groups, dtype, wtype):
    """dx is off by the errors of its two sums (48 u of their terms), of xh and of three products; dw and db by 64 u of
    the magnitudes of their terms for every 32 rows of a worker, its rows being added one after the other, and the slots
    after that."""
    per = -(-rows // groups)
    x, w, _, dy = inputs(rows, dim, groups, dtype, wtype, seed=1)
    _, m, r = layer_norm(x.double(), None, None, EPS, per)
    m, r = m.float(), r.float()
    norm = binding.make_norm(rows, dim, per, EPS, dtype, wtype)
    ws = binding.make_norm_workspace(norm)
    ws[256:].fill_(255)  # NaN in every slot
    dx, dw, db = torch.full_like(x, float("nan")), torch.full_like(w, float("nan")), torch.full_like(w, float("nan"))
    binding.sparsp_layer_norm_bwd(norm, dy, x, w, m, r, dx, dw, db, ws)
    X, W, DY, M, R = x.double(), w.double(), dy.double(), m.double(), r.double()
    want, want_w, want_b = layer_norm_back(DY, X, W, M, R, per, groups)
    g = torch.arange(rows, device="cuda") // per
    xh = ((X - M[:, None]) * R[:, None]).abs()
    exh = 3 * F32 * (xh + (X.abs() + M[:, None].abs()) * R[:, None])  # of xh
    a = (DY * W[g]).abs()
    c0 = 52 * F32 * a.mean(1, keepdim=True)
    c1 = (a * exh + 54 * F32 * a * xh).mean(1, keepdim=True)
    off = R[:, None] * (4 * F32 * a + c0 + xh * c1 + (exh + 4 * F32 * xh) * (a * xh).mean(1, keepdim=True)) + 4 * F32 * want.abs()
    close(dx, want, off + UNIT[dtype] * (want.abs() + off) + TINY[dtype], "dx")
    n = min(rows, 64 + rows // 148)
    size = torch.zeros_like(W).index_add_(0, g, DY.abs() * (xh + exh / F32 / n)), torch.zeros_like(W).index_add_(0, g, DY.abs())
    for got, ref, s, what in ((dw, want_w, size[0], "dw"), (db, want_b, size[1], "db")):
        off = (n + 20) * F32 * s
        close(got, ref, off + UNIT[wtype] * (ref.abs() + off) + TINY[wtype], what)
    # the same again, in place of dy: the same bits
    dx2, dw2, db2 = dy.clone(), torch.empty_like(w), torch.empty_like(w)
    binding.sparsp_layer_norm_bwd(norm, dx2, x, w, m, r, dx2, dw2, db2, ws)
    assert torch.equal(dx2, dx) and torch.equal(dw2, dw) and torch.equal(db2, db)


def test_without_weights_and_without_their_gradients():
    x, w, b, dy = inputs(37, 264, 1, BF, BF)
    norm = binding.make_norm(37, 264)
    y = torch.empty_like(x)
    mean, rstd = torch.empty(37, device="cuda"), torch.empty(37, device="cuda")
    binding.sparsp_layer_norm_fwd(norm, x, None, None, y, mean, rstd)
    want, m, r = layer_norm(x.double(), None, None, EPS, 37)
    close(y, want, fwd_bounds(x.double(), None, want, m, r, 37, BF)[0], "y")
    ones = torch.ones_like(w)
    dx, dx1, ws = torch.empty_like(x), torch.empty_like(x), binding.make_norm_workspace(norm)
    dw, dw1, db1 = torch.empty_like(w), torch.empty_like(w), torch.empty_like(w)
    binding.sparsp_layer_norm_bwd(norm, dy, x, None, mean, rstd, dx, None, None, None)
    binding.sparsp_layer_norm_bwd(norm, dy, x, ones, mean, rstd, dx1, dw1, db1, ws)
    assert torch.equal(dx, dx1)
    binding.sparsp_layer_norm_bwd(norm, dy, x, None, mean, rstd, dx, dw, None, ws)
    assert torch.equal(dw, dw1)


@pytest.mark.parametrize("dim,dtype", [(96, BF), (1100, BF), (77, FL)])
def test_strides_and_alignment(dim, dtype):
    """Rows with gaps, and a first row on an odd element: the gaps keep what they hold."""
    rows = 19
    x, w, b, dy = inputs(rows, dim, 1, dtype, dtype)
    for pad, shift in ((8, 0), (3, 0), (8, 1)):
        hold = [torch.full((rows * (dim + pad) + shift,), 7.0, dtype=dtype, device="cuda") for _ in range(4)]
        view = [h[shift:].view(rows, dim + pad)[:, :dim] for h in hold]
        view[0].copy_(x)
        view[2].copy_(dy)
        norm = binding.make_norm(rows, dim, 0, EPS, dtype, dtype, stride_x=dim + pad, stride_y=dim + pad)
        mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        binding.sparsp_layer_norm_fwd(norm, view[0], w, b, view[1], mean, rstd)
        want, m, r = layer_norm(x.double(), w.double(), b.double(), EPS, rows)
        close(view[1], want, fwd_bounds(x.double(), w.double(), want, m, r, rows, dtype)[0], "y")
        ws, dw, db = binding.make_norm_workspace(norm), torch.empty_like(w), torch.empty_like(b)
        binding.sparsp_layer_norm_bwd(norm, view[2], view[0], w, mean, rstd, view[3], dw, db, ws)
        full = binding.make_norm(rows, dim, 0, EPS, dtype, dtype)
        dx = torch.empty_like(x)
        binding.sparsp_layer_norm_bwd(full, dy, x, w, mean, rstd, dx, dw, db, ws)
        # other vectors, other order of additions: within a step of the type, or of fp32 sums
        off = UNIT[dtype] * 2 * dx.double().abs() + 200 * F32 * (dx.double().abs().amax(1, keepdim=True) + 1)
        close(view[3], dx, off, "dx")
        for h in hold:
            gap = torch.ones_like(h, dtype=torch.bool)
            gap[shift:].view(rows, dim + pad)[:, :dim] = False
            assert bool((h[gap] == 7.0).all())


def test_large_offset_loses_nothing():
    """A mean a thousand times the spread: deviations are taken before they are squared."""
    x, w, b, _ = inputs(33, 4096, 1, FL, FL, offset=3000.0)
    norm = binding.make_norm(33, 4096, 0, EPS, FL, FL)
    y = torch.empty_like(x)
    binding.sparsp_layer_norm_fwd(norm, x, w, b, y, None, None)
    want, m, r = layer_norm(x.double(), w.double(), b.double(), EPS, 33)
    close(y, want, fwd_bounds(x.double(), w.double(), want, m, r, 33, FL)[0], "y")


def test_rows_of_equal_and_of_special_values():
    x = torch.randn(6, 320, generator=torch.Generator().manual_seed(0)).to(BF)
    x[0] = 0.0
    x[1] = 3.0
    x[2, 5] = float("nan")
    x[3, 7] = float("inf")
    x = x.cuda()
    w, b = torch.full((1, 320), 2.0, device="cuda"), torch.full((1, 320), 0.25, device="cuda")
    y = torch.empty_like(x)
    binding.sparsp_layer_norm_fwd(binding.make_norm(6, 320, weight_dtype=FL), x, w, b, y, None, None)
    assert bool((y[:2] == 0.25).all())
    assert bool(torch.isnan(y[2]).all()) and bool(torch.isnan(y[3]).all())
    assert bool(torch.isfinite(y[4:]).all())


def test_no_rows():
    norm = binding.make_norm(0, 64)
    none = torch.empty(0, 64, dtype=BF, device="cuda")
    binding.sparsp_layer_norm_fwd(norm, none, None, None, none, None, None)
    dw, db = (torch.full((1, 64), 9.0, dtype=BF, device="cuda") for _ in range(2))
    binding.sparsp_layer_norm_bwd(norm, none, none, None, None, None, none, dw, db, binding.make_norm_workspace(norm))
    assert bool((dw == 0).all()) and bool((db == 0).all())


@pytest.mark.parametrize("rows,dim,groups", [(6, 40, 1), (9, 1056, 3)])
def test_gradients_against_differences(rows, dim, groups):
    """L = sum g y in 64 bits; central differences along random directions, step 1e-5: off by their own third-order term
    (below 1e-7 of the terms' size) and by the kernel's fp32 sums."""
    per = rows // groups
    x, w, b, dy = inputs(rows, dim, groups, FL, FL, seed=4)
    norm = binding.make_norm(rows, dim, per, EPS, FL, FL)
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    binding.sparsp_layer_norm_fwd(norm, x, w, b, y, mean, rstd)
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    binding.sparsp_layer_norm_bwd(norm, dy, x, w, mean, rstd, dx, dw, db, binding.make_norm_workspace(norm))
    gen, step = torch.Generator().manual_seed(8), 1e-5
    base = [t.double() for t in (x, w, b)]
    for which, grad in ((0, dx), (1, dw), (2, db)):
        v = torch.randn(base[which].shape, generator=gen).double().cuda()
        loss = []
        for sign in (1, -1):
            args = [t + sign * step * v if i == which else t for i, t in enumerate(base)]
            loss.append((layer_norm(*args, EPS, per)[0] * dy.double()).sum())
        slope = float(loss[0] - loss[1]) / (2 * step)
        size = float((grad.double() * v).abs().sum())
        assert abs(slope - float((grad.double() * v).sum())) <= 1e-5 * size
