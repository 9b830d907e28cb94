"""Gated feed-forward against the plain 64-bit form.

Bounds: a sum of K products of 16-bit values in fp32, added 16 at a time, is off by at most (K / 16 + 8) 2^-23 of the sum
of the products' magnitudes (additions may cut instead of rounding).  The activations are within 2^-20 of |x|, their
slopes within 2^-20; |a'| <= 1.13.  dG and dU are rounded to 16 bits before they are multiplied: half a step of each."""
import pytest
import torch

from layer_reference import TINY, UNIT, activation, close
from paper_2609_32197_b200 import binding

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def inputs(m, d, f, dtype, seed=0):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(m, d, generator=gen).to(dtype).cuda()
    wg, wu = ((torch.randn(f, d, generator=gen) * 1.5 * d ** -0.5).to(dtype).cuda() for _ in range(2))
    dh = torch.randn(m, f, generator=gen).to(dtype).cuda()
    return x, wg, wu, dh


def acc(k):
    return (k / 16 + 8) * 2.0 ** -23


def check_forward(kind, dtype, x, wg, wu, h, gate, up):
    X, G, U = x.double(), wg.double(), wu.double()
    g, u = X @ G.T, X @ U.T
    eg, eu = acc(X.shape[1]) * (X.abs() @ G.abs().T), acc(X.shape[1]) * (X.abs() @ U.abs().T)
    a, _ = activation(kind, g)
    ea = 1.13 * eg + 2.0 ** -20 * g.abs()
    want = a * u
    off = ea * u.abs() + (a.abs() + ea) * eu
    close(h, want, off + UNIT[dtype] * (want.abs() + off) + TINY[dtype], "h")
    if gate is not None:
        close(gate, g, eg + UNIT[dtype] * (g.abs() + eg) + TINY[dtype], "gate")
        close(up, u, eu + UNIT[dtype] * (u.abs() + eu) + TINY[dtype], "up")


def check_backward(kind, dtype, dh, x, wg, wu, gate, up, dx, dwg, dwu):
    DH, X, G, U = dh.double(), x.double(), wg.double(), wu.double()
    a, slope = activation(kind, gate.double())
    dg, du = DH * up.double() * slope, DH * a
    eg = UNIT[dtype] * dg.abs() * 1.01 + 2.0 ** -19 * (DH * up.double()).abs() + TINY[dtype]
    eu = UNIT[dtype] * du.abs() * 1.01 + 2.0 ** -19 * (DH * gate.double()).abs() + TINY[dtype]
    m, f = DH.shape
    if dx is not None:
        want = dg @ G + du @ U
        off = eg @ G.abs() + eu @ U.abs() + acc(2 * f) * (dg.abs() @ G.abs() + du.abs() @ U.abs())
        close(dx, want, off + UNIT[dtype] * (want.abs() + off) + TINY[dtype], "dX")
    if dwg is not None:
        for got, d, e, what in ((dwg, dg, eg, "dWgate"), (dwu, du, eu, "dWup")):
            want = d.T @ X
            off = e.T @ X.abs() + acc(m) * (d.abs().T @ X.abs())
            close(got, want, off + UNIT[dtype] * (want.abs() + off) + TINY[dtype], what)


SHAPES = [
    # tokens, dim, hidden
    (1, 8, 8), (1, 64, 128), (1, 1000, 264), (2, 64, 16), (17, 72, 136), (77, 264, 120), (128, 64, 128), (129, 128, 256),
    (256, 192, 128), (257, 320, 392), (300, 1096, 72), (511, 40, 1032), (640, 256, 640), (1003, 584, 520), (5, 2048, 2056),
    (2500, 64, 72), (700, 2600, 3000),
]


@pytest.mark.parametrize("m,d,f", SHAPES)
@pytest.mark.parametrize("kind,dtype", [("silu", BF), ("gelu_tanh", HF), ("gelu", BF)])
def test_forward(m, d, f, kind, dtype):
    x, wg, wu, _ = inputs(m, d, f, dtype)
    ffn = binding.make_ffn(m, d, f, kind, dtype)
    ws = binding.make_ffn_workspace(ffn, backward=False)
    ws[256:].fill_(255)  # NaN in every partial sum
    h, gate, up = (torch.full((m, f), float("nan"), dtype=dtype, device="cuda") for _ in range(3))
    binding.sparsp_gated_ffn_fwd(ffn, x, wg, wu, h, gate, up, ws)
    assert binding.sparsp_status(ws) == binding.SPARSP_OK
    check_forward(kind, dtype, x, wg, wu, h, gate, up)
    alone = torch.full_like(h, float("nan"))
    binding.sparsp_gated_ffn_fwd(ffn, x, wg, wu, alone, None, None, ws)
    assert torch.equal(alone, h)


@pytest.mark.parametrize("m,d,f", SHAPES)
@pytest.mark.parametrize("kind,dtype", [("silu", BF), ("gelu_tanh", BF), ("gelu", HF)])
def test_backward(m, d, f, kind, dtype):
    x, wg, wu, dh = inputs(m, d, f, dtype, seed=1)
    gate, up = x @ wg.T, x @ wu.T
    ffn = binding.make_ffn(m, d, f, kind, dtype)
    ws = binding.make_ffn_workspace(ffn)
    ws[256:].fill_(255)
    dx = torch.full_like(x, float("nan"))
    dwg, dwu = torch.full_like(wg, float("nan")), torch.full_like(wu, float("nan"))
    binding.sparsp_gated_ffn_bwd(ffn, dh, x, wg, wu, gate, up, dx, dwg, dwu, ws)
    assert binding.sparsp_status(ws) == binding.SPARSP_OK
    check_backward(kind, dtype, dh, x, wg, wu, gate, up, dx, dwg, dwu)
    # each half alone: the same bits
    dx2, dwg2, dwu2 = torch.empty_like(dx), torch.empty_like(dwg), torch.empty_like(dwu)
    binding.sparsp_gated_ffn_bwd(ffn, dh, None, wg, wu, gate, up, dx2, None, None, ws)
    binding.sparsp_gated_ffn_bwd(ffn, dh, x, None, None, gate, up, None, dwg2, dwu2, ws)
    assert torch.equal(dx2, dx) and torch.equal(dwg2, dwg) and torch.equal(dwu2, dwu)


def test_strides_and_interleaved_weights():
    """Wgate and Wup as alternating rows of one matrix, padded rows elsewhere; the gaps keep what they hold."""
    m, d, f, dtype = 140, 200, 264, BF
    x0, wg0, wu0, dh0 = inputs(m, d, f, dtype, seed=2)
    both = torch.stack((wg0, wu0), 1).contiguous()  # [f][2][d]
    wg, wu = both[:, 0], both[:, 1]
    hold = torch.full((m, d + 24), 7.0, dtype=dtype, device="cuda")
    x = hold[:, :d]
    x.copy_(x0)
    wide = [torch.full((m, f + 40), 7.0, dtype=dtype, device="cuda") for _ in range(4)]
    h, gate, up, dh = (t[:, :f] for t in wide)
    dh.copy_(dh0)
    ffn = binding.make_ffn(m, d, f, "silu", dtype, stride_x=d + 24, stride_h=f + 40, stride_w=2 * d)
    ws = binding.make_ffn_workspace(ffn)
    binding.sparsp_gated_ffn_fwd(ffn, x, wg, wu, h, gate, up, ws)
    check_forward("silu", dtype, x0, wg0, wu0, h, gate, up)
    hold_dx, grads = torch.full((m, d + 24), 7.0, dtype=dtype, device="cuda"), torch.empty_like(both)
    binding.sparsp_gated_ffn_bwd(ffn, dh, x, wg, wu, gate, up, hold_dx, grads[:, 0], grads[:, 1], ws)
    check_backward("silu", dtype, dh0, x0, wg0, wu0, gate, up, hold_dx[:, :d], grads[:, 0], grads[:, 1])
    assert binding.sparsp_status(ws) == binding.SPARSP_OK
    for t, n in [(w, f) for w in wide] + [(hold, d), (hold_dx, d)]:
        assert bool((t[:, n:] == 7.0).all())


def test_no_tokens():
    ffn = binding.make_ffn(0, 64, 72)
    ws, none = binding.make_ffn_workspace(ffn), torch.empty(0, 72, dtype=BF, device="cuda")
    binding.sparsp_gated_ffn_fwd(ffn, none, none, none, none, None, None, ws)
    dwg, dwu = (torch.full((72, 64), 9.0, dtype=BF, device="cuda") for _ in range(2))
    binding.sparsp_gated_ffn_bwd(ffn, none, none, none, none, none, none, none, dwg, dwu, ws)
    assert bool((dwg == 0).all()) and bool((dwu == 0).all())


@pytest.mark.parametrize("kind", ["silu", "gelu_tanh", "gelu"])
def test_projections_of_every_size(kind):
    """Gates far out on both sides: the activation goes to 0 or to its argument, its slope to 0 or 1, nothing to NaN."""
    m, d, f = 64, 64, 64
    x = torch.zeros(m, d, dtype=BF, device="cuda")
    x[torch.arange(m), torch.arange(d)] = 1.0
    size = torch.tensor([0.0, 1e-30, 1e-3, 0.5, 3.0, 9.0, 30.0, 88.0, 104.0, 1e4, 1e19, 3e38], dtype=torch.float64)
    vals = torch.cat((size, -size)).repeat(3)[:d].to(BF).cuda()
    wg = vals[None, :].expand(f, d).contiguous()
    wu = torch.ones(f, d, dtype=BF, device="cuda")
    ffn = binding.make_ffn(m, d, f, kind)
    ws = binding.make_ffn_workspace(ffn)
    h, gate, up = (torch.empty(m, f, dtype=BF, device="cuda") for _ in range(3))
    binding.sparsp_gated_ffn_fwd(ffn, x, wg, wu, h, gate, up, ws)
    assert torch.equal(gate, vals[:, None].expand(m, f))
    a, _ = activation(kind, vals[:, None].double().clamp(-1e30, 1e30))
    a = torch.where(vals[:, None].double() < -1e9, torch.zeros_like(a), a)
    a = torch.where(vals[:, None].double() > 1e9, vals[:, None].double(), a).expand(m, f)
    close(h, a, UNIT[BF] * a.abs() * 1.01 + 2.0 ** -20 * vals[:, None].double().abs().clamp(max=100.0) + 1e-38, "h")
    dh = torch.ones(m, f, dtype=BF, device="cuda")
    dx, dwg, dwu = torch.empty_like(x), torch.empty_like(wg), torch.empty_like(wu)
    # X = I: dW is dG and dU themselves, transposed
    binding.sparsp_gated_ffn_bwd(ffn, dh, x, wg, wu, gate, up, dx, dwg, dwu, ws)
    assert bool(torch.isfinite(dwg).all())
    big = vals.double().abs() > 50
    close(dwg[0][big], (vals.double()[big] > 0).double(), torch.tensor(2.0 ** -19, device="cuda"), "slope")


def test_special_values_stay_in_their_rows():
    x, wg, wu, _ = inputs(200, 136, 72, BF)
    clean = torch.empty(200, 72, dtype=BF, device="cuda")
    ffn = binding.make_ffn(200, 136, 72)
    ws = binding.make_ffn_workspace(ffn, backward=False)
    binding.sparsp_gated_ffn_fwd(ffn, x, wg, wu, clean, None, None, ws)
    x[3, 5], x[150, 135] = float("nan"), float("inf")
    h = torch.empty_like(clean)
    binding.sparsp_gated_ffn_fwd(ffn, x, wg, wu, h, None, None, ws)
    rows = torch.ones(200, dtype=torch.bool, device="cuda")
    rows[[3, 150]] = False
    assert torch.equal(h[rows], clean[rows])
    assert bool(torch.isnan(h[3]).all()) and not bool(torch.isfinite(h[150]).all())


@pytest.mark.parametrize("m,d,f", [(33, 72, 136), (300, 128, 264)])
def test_calls_agree_bit_for_bit(m, d, f):
    """Split sums are added in one order whatever runs when, and results do not depend on rows beside them."""
    x, wg, wu, dh = inputs(m, d, f, BF, seed=3)
    ffn = binding.make_ffn(m, d, f)
    ws = binding.make_ffn_workspace(ffn)
    first = None
    for _ in range(20):
        h, gate, up = (torch.empty(m, f, dtype=BF, device="cuda") for _ in range(3))
        dx, dwg, dwu = torch.empty_like(x), torch.empty_like(wg), torch.empty_like(wu)
        binding.sparsp_gated_ffn_fwd(ffn, x, wg, wu, h, gate, up, ws)
        binding.sparsp_gated_ffn_bwd(ffn, dh, x, wg, wu, gate, up, dx, dwg, dwu, ws)
        got = [t.clone() for t in (h, gate, up, dx, dwg, dwu)]
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(first, got))


@pytest.mark.parametrize("kind", ["silu", "gelu_tanh", "gelu"])
def test_gradients_against_differences(kind):
    """L = sum dh a(X Wg^T) (X Wu^T) in 64 bits, central differences with step 1e-5 along random directions; the kernel
    takes gate and up in 16 bits and rounds dG, dU and its results, each by half a step of magnitudes that add up."""
    m, d, f = 150, 96, 200
    x, wg, wu, dh = inputs(m, d, f, HF, seed=5)
    ffn = binding.make_ffn(m, d, f, kind, HF)
    ws = binding.make_ffn_workspace(ffn)
    h, gate, up = (torch.empty(m, f, dtype=HF, device="cuda") for _ in range(3))
    binding.sparsp_gated_ffn_fwd(ffn, x, wg, wu, h, gate, up, ws)
    dx, dwg, dwu = torch.empty_like(x), torch.empty_like(wg), torch.empty_like(wu)
    binding.sparsp_gated_ffn_bwd(ffn, dh, x, wg, wu, gate, up, dx, dwg, dwu, ws)
    base, gen, step = [t.double() for t in (x, wg, wu)], torch.Generator().manual_seed(6), 1e-5
    a, slope = activation(kind, base[0] @ base[1].T)
    DH, U = dh.double().abs(), (base[0] @ base[2].T).abs()
    dg, du = DH * U * (slope.abs() + 1), DH * (a.abs() + 1)
    for which, grad in ((0, dx), (1, dwg), (2, dwu)):
        v = torch.randn(base[which].shape, generator=gen).double().cuda()
        loss = []
        for sign in (1, -1):
            X, G, W = (t + sign * step * v if i == which else t for i, t in enumerate(base))
            loss.append((dh.double() * activation(kind, X @ G.T)[0] * (X @ W.T)).sum())
        slope_v = float(loss[0] - loss[1]) / (2 * step)
        size = dg @ base[1].abs() + du @ base[2].abs() if which == 0 else (dg if which == 1 else du).T @ base[0].abs()
        assert abs(slope_v - float((grad.double() * v).sum())) <= 4 * UNIT[HF] * float((size * v.abs()).sum())
