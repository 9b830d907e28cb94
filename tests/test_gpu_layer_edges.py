"""The token-wise operators where their work is shared out differently: rows in classes, few rows, groups smaller than a
class, tiles whose K is shared, few tokens, and calls between the caller's own kernels.  Bounds as in the operators' own
tests."""
import pytest
import torch

import test_gpu_gated_ffn as ffn_tests
from layer_reference import F32, TINY, UNIT, close, layer_norm, layer_norm_back
from paper_2609_32197_b200 import binding
from test_gpu_layer_norm import EPS, fwd_bounds, inputs

pytestmark = pytest.mark.gpu
BF, HF, FL = torch.bfloat16, torch.float16, torch.float32


def check_norm(x, w, b, dy, per, groups, norm, y, dx):
    rows, dim, dtype, wtype = *x.shape, x.dtype, w.dtype
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    binding.sparsp_layer_norm_fwd(norm, x, w, b, y, mean, rstd)
    want, m, r = layer_norm(x.double(), w.double(), b.double(), EPS, per)
    by, bm, br = fwd_bounds(x.double(), w.double(), want, m, r, per, dtype)
    close(y, want, by, "y")
    close(mean, m, bm, "mean")
    close(rstd, r, br, "rstd")
    ws = binding.make_norm_workspace(norm)
    ws[256:].fill_(255)
    dw, db = torch.full_like(w, float("nan")), torch.full_like(w, float("nan"))
    binding.sparsp_layer_norm_bwd(norm, dy, x, w, mean, rstd, dx, dw, db, ws)
    X, W, DY, M, R = x.double(), w.double(), dy.double(), mean.double(), rstd.double()
    want, want_w, want_b = layer_norm_back(DY, X, W, M, R, per, groups)
    g = torch.arange(rows, device="cuda") // per
    xh = ((X - M[:, None]) * R[:, None]).abs()
    exh = 3 * F32 * (xh + (X.abs() + M[:, None].abs()) * R[:, None])
    a = (DY * W[g]).abs()
    c0, c1 = 52 * F32 * a.mean(1, keepdim=True), (a * exh + 54 * F32 * a * xh).mean(1, keepdim=True)
    off = R[:, None] * (4 * F32 * a + c0 + xh * c1 + (exh + 4 * F32 * xh) * (a * xh).mean(1, keepdim=True)) + 4 * F32 * want.abs()
    close(dx, want, off + UNIT[dtype] * (want.abs() + off) + TINY[dtype], "dx")
    n = min(rows, 64 + rows // 148)
    for got, ref, terms, what in ((dw, want_w, DY.abs() * (xh + exh / F32 / n), "dw"), (db, want_b, DY.abs(), "db")):
        off = (n + 20) * F32 * torch.zeros_like(W).index_add_(0, g, terms)
        close(got, ref, off + UNIT[wtype] * (ref.abs() + off) + TINY[wtype], what)


@pytest.mark.parametrize("dtype", [BF, HF, FL])
@pytest.mark.parametrize("dim", [2, 7, 9, 31, 33, 63, 64, 65, 100, 127, 129, 250, 255, 257, 263, 505, 511, 513, 1021, 2045, 2050])
def test_widths_around_every_edge(dim, dtype):
    for rows, groups in ((1, 1), (3, 3), (5, 1), (13, 5), (97, 4), (2500, 3)):
        if rows * dim > 1500000:
            continue
        per = -(-rows // groups)
        groups = -(-rows // per)
        x, w, b, dy = inputs(rows, dim, groups, dtype, FL, seed=rows)
        norm = binding.make_norm(rows, dim, per, EPS, dtype, FL)
        check_norm(x, w, b, dy, per, groups, norm, torch.full_like(x, float("nan")), torch.full_like(x, float("nan")))


@pytest.mark.parametrize("dtype,dim", [(BF, 5113), (BF, 5127), (HF, 8185), (HF, 8193), (FL, 4999), (FL, 8189), (BF, 16383),
                                       (FL, 9001)])
def test_long_rows_of_odd_length(dtype, dim):
    x, w, b, dy = inputs(19, dim, 2, dtype, dtype, seed=3)
    norm = binding.make_norm(19, dim, 10, EPS, dtype, dtype)
    check_norm(x, w, b, dy, 10, 2, norm, torch.full_like(x, float("nan")), torch.full_like(x, float("nan")))


@pytest.mark.parametrize("dtype,dim,pad_x,pad_y", [(BF, 70, 2, 10), (BF, 70, 2, 3), (FL, 1000, 1, 5), (FL, 1000, 1, 2),
                                                    (HF, 300, 4, 4), (BF, 5121, 3, 3)])
def test_rows_with_gaps_of_their_own(dtype, dim, pad_x, pad_y):
    """x and y with different gaps: rows that begin alike, and rows that do not; nothing outside the rows changes."""
    rows = 41
    x, w, b, dy = inputs(rows, dim, 1, dtype, dtype, seed=5)
    hold = [torch.full((rows, dim + p), 7.0, dtype=dtype, device="cuda") for p in (pad_x, pad_y, pad_y, pad_x)]
    vx, vy, vdy, vdx = (h[:, :dim] for h in hold)
    vx.copy_(x)
    vdy.copy_(dy)
    norm = binding.make_norm(rows, dim, 0, EPS, dtype, dtype, stride_x=dim + pad_x, stride_y=dim + pad_y)
    check_norm(vx, w, b, vdy, rows, 1, norm, vy, vdx)
    assert all(bool((h[:, dim:] == 7.0).all()) for h in hold)


@pytest.mark.parametrize("m,d,f", [
    (3, 328, 9600), (17, 136, 4800), (33, 72, 2400), (100, 1992, 2368), (127, 64, 9480),  # few tokens, every tile height
    (512, 4096, 2048), (300, 4096, 5000), (200, 10240, 6400),  # forward: a last round shared out, in both ways
])
def test_forward_shared_out(m, d, f):
    x, wg, wu, _ = ffn_tests.inputs(m, d, f, BF, seed=7)
    ffn = binding.make_ffn(m, d, f, "silu", BF)
    ws = binding.make_ffn_workspace(ffn, backward=False)
    ws[256:].fill_(255)
    h, gate, up = (torch.full((m, f), float("nan"), dtype=BF, device="cuda") for _ in range(3))
    before = binding.sparsp_launch_count()
    binding.sparsp_gated_ffn_fwd(ffn, x, wg, wu, h, gate, up, ws)
    assert binding.sparsp_launch_count() - before == (1 if m <= 128 else 2)
    assert binding.sparsp_status(ws) == binding.SPARSP_OK
    ffn_tests.check_forward("silu", BF, x, wg, wu, h, gate, up)


@pytest.mark.parametrize("m,d,f", [(1003, 1160, 2504), (9, 600, 4000), (2100, 1304, 1504), (4100, 264, 520), (130, 2600, 5000),
                                   (5000, 1032, 3080)])
def test_backward_shared_out(m, d, f):
    """dX and dW in one launch or one after the other, whole tiles and shared ones."""
    x, wg, wu, dh = ffn_tests.inputs(m, d, f, BF, seed=8)
    gate, up = x @ wg.T, x @ wu.T
    ffn = binding.make_ffn(m, d, f, "silu", BF)
    ws = binding.make_ffn_workspace(ffn)
    ws[256:].fill_(255)
    dx, dwg, dwu = (torch.full_like(t, float("nan")) for t in (x, wg, wu))
    binding.sparsp_gated_ffn_bwd(ffn, dh, x, wg, wu, gate, up, dx, dwg, dwu, ws)
    assert binding.sparsp_status(ws) == binding.SPARSP_OK
    ffn_tests.check_backward("silu", BF, dh, x, wg, wu, gate, up, dx, dwg, dwu)
    dx2, dwg2, dwu2 = torch.empty_like(dx), torch.empty_like(dwg), torch.empty_like(dwu)
    binding.sparsp_gated_ffn_bwd(ffn, dh, None, wg, wu, gate, up, dx2, None, None, ws)
    binding.sparsp_gated_ffn_bwd(ffn, dh, x, None, None, gate, up, None, dwg2, dwu2, ws)
    assert torch.equal(dx2, dx) and torch.equal(dwg2, dwg) and torch.equal(dwu2, dwu)


def test_between_the_callers_own_kernels():
    """Inputs written right before a call and outputs read and overwritten right after it, on a stream of the caller's."""
    m, d, f = 260, 264, 520
    x0, wg, wu, dh = ffn_tests.inputs(m, d, f, BF, seed=9)
    ffn, norm = binding.make_ffn(m, d, f), binding.make_norm(m, d)
    ws, nws = binding.make_ffn_workspace(ffn), binding.make_norm_workspace(norm)
    w = torch.ones(1, d, dtype=BF, device="cuda")

    def chain(x):
        n, mean, rstd = torch.empty_like(x), torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
        h, gate, up = (torch.empty(m, f, dtype=BF, device="cuda") for _ in range(3))
        dx, dwg, dwu, dn, dw, db = (torch.empty_like(t) for t in (x, wg, wu, x, w, w))
        z = x * 1.0
        binding.sparsp_layer_norm_fwd(norm, z, w, w, n, mean, rstd)
        z.zero_()
        n2 = n + 0
        n.zero_()
        binding.sparsp_gated_ffn_fwd(ffn, n2, wg, wu, h, gate, up, ws)
        g2, u2 = gate + 0, up + 0
        gate.zero_()
        up.zero_()
        binding.sparsp_gated_ffn_bwd(ffn, dh, n2, wg, wu, g2, u2, dx, dwg, dwu, ws)
        g2.zero_()
        n2.zero_()
        dx2 = dx + 0
        dx.zero_()
        z.copy_(x)
        binding.sparsp_layer_norm_bwd(norm, dx2, z, w, mean, rstd, dn, dw, db, nws)
        dx2.zero_()
        return [t + 0 for t in (h, dwg, dwu, dn, dw, db)]

    want = []
    for k in range(3):
        want.append(chain(x0 * (k + 1)))
        torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(10):
            for k in range(3):
                got = chain(x0 * (k + 1))
                assert all(torch.equal(a, b) for a, b in zip(got, want[k]))
    torch.cuda.current_stream().wait_stream(side)


@pytest.mark.parametrize("m,d,f", [(1, 64, 128), (2, 88, 936), (64, 264, 72), (128, 600, 520), (100, 2600, 200)])
@pytest.mark.parametrize("kind,dtype", [("silu", BF), ("gelu", HF)])
def test_few_tokens_keep_what_the_operands_round_off(m, d, f, kind, dtype):
    """Up to 128 tokens dG and dU are in two parts: off by the square of a rounding, and by what a(x) and a'(x) are."""
    x, wg, wu, dh = ffn_tests.inputs(m, d, f, dtype, seed=11)
    gate, up = x @ wg.T, x @ wu.T
    ffn = binding.make_ffn(m, d, f, kind, dtype)
    ws = binding.make_ffn_workspace(ffn)
    ws[256:].fill_(255)
    dx, dwg, dwu = (torch.full_like(t, float("nan")) for t in (x, wg, wu))
    binding.sparsp_gated_ffn_bwd(ffn, dh, x, wg, wu, gate, up, dx, dwg, dwu, ws)
    assert binding.sparsp_status(ws) == binding.SPARSP_OK
    DH, X, G, U = (t.double() for t in (dh, x, wg, wu))
    a, slope = ffn_tests.activation(kind, gate.double())
    dg, du = DH * up.double() * slope, DH * a
    eg = 2 * UNIT[dtype] ** 2 * dg.abs() + 2.0 ** -19 * (DH * up.double()).abs() + TINY[dtype]
    eu = 2 * UNIT[dtype] ** 2 * du.abs() + 2.0 ** -19 * (DH * gate.double()).abs() + TINY[dtype]
    want = dg @ G + du @ U
    off = eg @ G.abs() + eu @ U.abs() + ffn_tests.acc(4 * f) * (dg.abs() @ G.abs() + du.abs() @ U.abs())
    close(dx, want, off + UNIT[dtype] * (want.abs() + off) + TINY[dtype], "dX")
    for got, t, e, what in ((dwg, dg, eg, "dWgate"), (dwu, du, eu, "dWup")):
        want = t.T @ X
        off = e.T @ X.abs() + ffn_tests.acc(2 * m) * (t.abs().T @ X.abs())
        close(got, want, off + UNIT[dtype] * (want.abs() + off) + TINY[dtype], what)


def test_infinite_gradients_of_few_tokens():
    """A dG past the type's range is an infinity, as rounding makes it; what it leaves is not NaN by itself."""
    m, d, f = 3, 64, 64
    x, wg, wu, dh = ffn_tests.inputs(m, d, f, HF, seed=12)
    gate, up = torch.full((m, f), 100.0, dtype=HF, device="cuda"), torch.full((m, f), 60000.0, dtype=HF, device="cuda")
    dh.fill_(1.0)
    dh[1] = 4.0  # 4 * 60000 * 1: infinite in 16 bits
    wg.fill_(1.0)
    ffn = binding.make_ffn(m, d, f, "silu", HF)
    ws = binding.make_ffn_workspace(ffn)
    dx, dwg, dwu = (torch.empty_like(t) for t in (x, wg, wu))
    binding.sparsp_gated_ffn_bwd(ffn, dh, x, wg, wu * 0, gate, up, dx, dwg, dwu, ws)
    assert bool(torch.isinf(dx[1]).all()) and not bool(torch.isnan(dx[1]).any())


@pytest.mark.parametrize("kind", ["silu", "gelu_tanh", "gelu"])
@pytest.mark.parametrize("m", [100, 300])
def test_activations_keep_their_relative_error(m, kind):
    """Gates from -6 to 3 as they are, each times powers of two: what is left of the activation far down shows.

    Off by: the argument of the exponential, up to 40 in size, with four roundings (160 * 2^-24 * ln 2 = 2^-17.2), a
    polynomial within 2^-20, six roundings; together below 2^-16.  Then one rounding to the type."""
    d, f = 64, 208
    x = torch.zeros(m, d, dtype=HF, device="cuda")
    x[:, 0], x[:, 1] = torch.linspace(-6, 3, m).to("cuda", HF), 1
    wg, wu = torch.zeros(f, d, dtype=HF, device="cuda"), torch.zeros(f, d, dtype=HF, device="cuda")
    wg[:, 0], wu[:, 1] = 1, 2.0 ** (torch.arange(f, device="cuda") % 13)
    h = torch.full((m, f), float("nan"), dtype=HF, device="cuda")
    ffn = binding.make_ffn(m, d, f, kind, HF)
    binding.sparsp_gated_ffn_fwd(ffn, x, wg, wu, h, None, None, binding.make_ffn_workspace(ffn, False))
    want = ffn_tests.activation(kind, x[:, :1].double())[0] * wu[None, :, 1].double()
    close(h, want, want.abs() * (UNIT[HF] + 2.0 ** -16) + TINY[HF], kind)


@pytest.mark.parametrize("dtype", [BF, FL])
@pytest.mark.parametrize("dim", [761, 768, 776, 1017, 1024, 1032, 1273, 1280, 1288, 1536, 1544, 2048, 2056, 2304, 2312, 2560, 2568,
                                 3079, 4096, 4104, 5120, 5128, 6144, 6152, 7680, 7688, 8192, 8200, 9216, 9224, 10240, 10248,
                                 12281, 12288, 12296, 16384])
def test_widths_where_another_worker_takes_over(dim, dtype):
    """Rows that just fit a worker, and that just do not; with classes, without, and value by value (a shifted tensor)."""
    for rows, groups, off in ((7, 2, 0), (211, 3, 0), (9, 1, 1)):
        per = -(-rows // groups)
        x, w, b, dy = inputs(rows, dim, groups, dtype, FL, seed=dim)
        base = torch.empty(rows * dim + off, dtype=dtype, device="cuda")
        base[off:] = x.flatten()
        norm = binding.make_norm(rows, dim, per, EPS, dtype, FL)
        check_norm(base[off:].view(rows, dim), w, b, dy, per, groups, norm, torch.full_like(x, float("nan")),
                   torch.full_like(x, float("nan")))


@pytest.mark.parametrize("dim", [40, 130, 640, 1152, 2048, 5120, 8192])
def test_few_rows_of_many_groups(dim):
    """Either side of where the weights' gradients are added in the launch that makes dx."""
    for per, groups in ((1, 1), (1, 7), (16, 8), (31, 1), (33, 1), (64, 5), (65, 2), (129, 1), (250, 2), (257, 1)):
        rows = per * groups
        x, w, b, dy = inputs(rows, dim, groups, BF, BF, seed=per)
        norm = binding.make_norm(rows, dim, per, EPS, BF, BF)
        check_norm(x, w, b, dy, per, groups, norm, torch.full_like(x, float("nan")), torch.full_like(x, float("nan")))


@pytest.mark.parametrize("most,m", [(200, 100), (129, 128), (255, 73), (300, 1)])
def test_a_workspace_for_more_tokens_serves_fewer(most, m):
    """The last, shorter batch in the workspace of the others: right, and nothing behind the workspace changes."""
    d, f = 264, 1000
    size = binding.sparsp_gated_ffn_workspace_bytes(binding.make_ffn(most, d, f), True)
    hold = torch.full((size + (4 << 20),), 77, dtype=torch.uint8, device="cuda")
    ws = hold[:size]
    ws[:256].zero_()
    x, wg, wu, dh = ffn_tests.inputs(m, d, f, BF, seed=13)
    gate, up = x @ wg.T, x @ wu.T
    ffn = binding.make_ffn(m, d, f)
    dx, dwg, dwu = (torch.full_like(t, float("nan")) for t in (x, wg, wu))
    binding.sparsp_gated_ffn_bwd(ffn, dh, x, wg, wu, gate, up, dx, dwg, dwu, ws)
    assert binding.sparsp_status(ws) == binding.SPARSP_OK
    ffn_tests.check_backward("silu", BF, dh, x, wg, wu, gate, up, dx, dwg, dwu)
    assert bool((hold[size:] == 77).all())


@pytest.mark.parametrize("rows", [1, 20, 5000])  # the weights' gradients in the launch that makes dx, and in one of their own
@pytest.mark.parametrize("per", [2 ** 62, 2 ** 63 - 1])
def test_one_group_said_as_a_huge_one(rows, per):
    dim = 264
    x, w, b, dy = inputs(rows, dim, 1, BF, BF, seed=21)
    check_norm(x, w, b, dy, rows, 1, binding.make_norm(rows, dim, per, EPS, BF, BF), torch.full_like(x, float("nan")),
               torch.full_like(x, float("nan")))


@pytest.mark.parametrize("m", [3, 100, 128, 200])
def test_infinite_operands_of_the_backward_pass(m):
    """An infinity in X or in the weights makes infinities where dG or dU is not zero, for few tokens too: what the first
    part's rounding left has either sign, or is zero, and must not make NaN of them."""
    d, f = 136, 264
    x, wg, wu, dh = ffn_tests.inputs(m, d, f, BF, seed=23)
    gate, up = x @ wg.T, x @ wu.T
    x[m // 2, 5], x[m - 1, 77] = float("inf"), -float("inf")
    wg[3, 9], wg[f - 1, 100], wu[70, 20] = float("inf"), -float("inf"), float("inf")
    ffn = binding.make_ffn(m, d, f)
    ws = binding.make_ffn_workspace(ffn)
    ws[256:].fill_(255)
    dx, dwg, dwu = (torch.full_like(t, float("nan")) for t in (x, wg, wu))
    binding.sparsp_gated_ffn_bwd(ffn, dh, x, wg, wu, gate, up, dx, dwg, dwu, ws)
    assert binding.sparsp_status(ws) == binding.SPARSP_OK
    assert bool(torch.isinf(dwg[:, 5]).all()) and bool(torch.isinf(dx[:, 20]).all())
    ffn_tests.check_backward("silu", BF, dh, x, wg, wu, gate, up, dx, dwg, dwu)


@pytest.mark.parametrize("m,d,f,together", [(64, 18432, 256, False), (3, 16640, 72, False), (64, 8192, 256, True),
                                            (128, 12288, 512, True), (129, 18432, 256, True)])
def test_one_launch_for_both_gradients_where_it_is_shorter(m, d, f, together):
    """Few tokens of a wide layer: in one launch dX would take nearly all multiprocessors from a dW of more tiles."""
    x, wg, wu, dh = ffn_tests.inputs(m, d, f, BF, seed=29)
    gate, up = x @ wg.T, x @ wu.T
    ffn = binding.make_ffn(m, d, f)
    ws = binding.make_ffn_workspace(ffn)
    ws[256:].fill_(255)
    dx, dwg, dwu = (torch.full_like(t, float("nan")) for t in (x, wg, wu))
    before = binding.sparsp_launch_count()
    binding.sparsp_gated_ffn_bwd(ffn, dh, x, wg, wu, gate, up, dx, dwg, dwu, ws)
    assert (binding.sparsp_launch_count() - before <= 3) == together
    assert binding.sparsp_status(ws) == binding.SPARSP_OK
    ffn_tests.check_backward("silu", BF, dh, x, wg, wu, gate, up, dx, dwg, dwu)
    dx2, dwg2, dwu2 = torch.empty_like(dx), torch.empty_like(dwg), torch.empty_like(dwu)
    binding.sparsp_gated_ffn_bwd(ffn, dh, None, wg, wu, gate, up, dx2, None, None, ws)
    binding.sparsp_gated_ffn_bwd(ffn, dh, x, None, None, gate, up, None, dwg2, dwu2, ws)
    assert torch.equal(dx2, dx) and torch.equal(dwg2, dwg) and torch.equal(dwu2, dwu)


@pytest.mark.parametrize("m,d,f,launches", [(512, 2048, 5120, 1), (250, 2048, 2560, 1), (512, 8192, 5120, 2), (250, 8192, 2560, 2),
                                            (256, 4096, 8192, 1), (256, 8192, 768, 2)])
def test_a_last_round_is_shared_out_where_that_is_shorter(m, d, f, launches):
    """Sums written, read and added by a launch of their own cost about as much as 16 to 40 blocks of K."""
    x, wg, wu, _ = ffn_tests.inputs(m, d, f, BF, seed=31)
    ffn = binding.make_ffn(m, d, f)
    ws = binding.make_ffn_workspace(ffn, backward=False)
    ws[256:].fill_(255)
    h, gate, up = (torch.full((m, f), float("nan"), dtype=BF, device="cuda") for _ in range(3))
    before = binding.sparsp_launch_count()
    binding.sparsp_gated_ffn_fwd(ffn, x, wg, wu, h, gate, up, ws)
    assert binding.sparsp_launch_count() - before == launches
    assert binding.sparsp_status(ws) == binding.SPARSP_OK
    ffn_tests.check_forward("silu", BF, x, wg, wu, h, gate, up)


@pytest.mark.parametrize("dtype,wtype", [(BF, BF), (BF, FL), (FL, FL), (HF, HF)])
@pytest.mark.parametrize("dim", [24, 333, 1152, 1921, 5120, 5127])
def test_many_groups(dim, dtype, wtype):
    """Weights per row or per few rows: groups that one worker has all of, groups across the parts of two and more, few
    slots of a group and many; in a workspace of just the size, with what lies behind it kept."""
    for per, groups in ((1, 3001), (2, 1501), (3, 1000), (7, 700), (20, 250), (61, 75), (200, 20), (900, 5)):
        rows = per * groups - (per > 2)  # the last group is smaller
        if rows * dim > 1 << 24:
            continue
        x, w, b, dy = inputs(rows, dim, groups, dtype, wtype, seed=per)
        norm = binding.make_norm(rows, dim, per, EPS, dtype, wtype)
        size = binding.sparsp_layer_norm_workspace_bytes(norm)
        hold = torch.full((size + (1 << 20),), 255, dtype=torch.uint8, device="cuda")
        mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        y, dx = torch.full_like(x, float("nan")), torch.full_like(x, float("nan"))
        binding.sparsp_layer_norm_fwd(norm, x, w, b, y, mean, rstd)
        dw, db = torch.full_like(w, float("nan")), torch.full_like(w, float("nan"))
        binding.sparsp_layer_norm_bwd(norm, dy, x, w, mean, rstd, dx, dw, db, hold[:size])
        assert bool((hold[size:] == 255).all())
        check_norm(x, w, b, dy, per, groups, norm, y, dx)
        check_weight_gradients(x, dy, mean, rstd, per, groups, dw, db)
        # one of the two wanted, gradients that do not begin on 16 bytes: the same values
        odd = torch.full((w.numel() + 1,), float("nan"), dtype=wtype, device="cuda")[1:].view_as(w)
        binding.sparsp_layer_norm_bwd(norm, dy, x, w, mean, rstd, dx, odd, None, hold[:size])
        assert torch.equal(odd, dw)
        binding.sparsp_layer_norm_bwd(norm, dy, x, w, mean, rstd, dx, None, odd, hold[:size])
        assert torch.equal(odd, db)


def check_weight_gradients(x, dy, mean, rstd, per, groups, dw, db):
    """Sums of a group's terms in fp32, by at most 32 + 60 additions in a row (a worker's rows, slots, lanes)."""
    X, DY, M, R = x.double(), dy.double(), mean.double()[:, None], rstd.double()[:, None]
    g = torch.arange(x.shape[0], device="cuda") // per
    xh = (X - M) * R
    of = lambda t: torch.zeros(groups, x.shape[1], dtype=torch.float64, device="cuda").index_add_(0, g, t)  # noqa: E731
    exh = 3 * F32 * (xh.abs() + (X.abs() + M.abs()) * R)
    terms = min(per, 900) + 8
    for got, want, off in ((dw, of(DY * xh), of(DY.abs() * exh + terms * F32 * (DY * xh).abs())),
                           (db, of(DY), of(terms * F32 * DY.abs()))):
        close(got, want, off + UNIT[got.dtype] * (want.abs() + off) + TINY[got.dtype], "weights' gradients")


@pytest.mark.parametrize("dim", [128, 1920, 1921])
def test_a_row_of_weights_per_row_takes_one_launch(dim):
    rows = 6000
    x, w, b, dy = inputs(rows, dim, rows, BF, BF, seed=1)
    norm = binding.make_norm(rows, dim, 1, EPS, BF, BF)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    y, dx, dw, db = (torch.empty_like(x) for _ in range(4))
    binding.sparsp_layer_norm_fwd(norm, x, w, b, y, mean, rstd)
    before = binding.sparsp_launch_count()
    binding.sparsp_layer_norm_bwd(norm, dy, x, w, mean, rstd, dx, dw, db, binding.make_norm_workspace(norm))
    assert binding.sparsp_launch_count() - before == 1
    xh = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    close(dw, dy.double() * xh, (UNIT[BF] + 8 * F32) * (dy.double() * xh).abs() + 8 * F32 * dy.double().abs() *
          (x.double().abs() + mean.double().abs()[:, None]) * rstd.double()[:, None], "dweight")
    assert torch.equal(db, dy)
