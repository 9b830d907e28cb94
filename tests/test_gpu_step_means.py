"""Rows whose mean is far from zero: what a norm keeps of them is their difference to the mean.

That difference is one fp32 operation, off by 2^-24 of itself, and the scale another: normed values are within 2 2^-24 of
themselves for the statistics that the call has, however large the mean is.  Everything else is as in step_reference.py."""
import pytest
import torch

import step_reference as ref
from layer_reference import F32 as U, close
from paper_2609_32197_b200 import binding
from test_gpu_gated_norm import BF, EPS, FL, HF, backward, check, forward, inputs, rounded, without

pytestmark = pytest.mark.gpu


def again(v, stats):
    m, r = stats.double()[:, :1], stats.double()[:, 1:]
    vh = (v - m) * r
    return vh, 2 * U * vh.abs() * ref.MORE


def check_normed(got, vh, evh, w, b, like, name):
    """got = vh w + b in one more operation"""
    w = torch.ones_like(vh) if w is None else w.double()
    b = torch.zeros_like(vh) if b is None else b.double()
    n = vh * w + b
    close(got, n, rounded(n, evh * w.abs() + U * (n.abs() + (vh * w).abs()), like), name)


def far_inputs(rows, dim, ratio, norm_y, norm_r, seed):
    """Deviations of about 1; gradients that go along with the rows, so that sums along a row do not cancel."""
    v = inputs(rows, dim, 1, FL, FL, seed)
    gen = torch.Generator().manual_seed(seed + 1)
    dx, dy = (torch.randn(rows, dim, generator=gen).cuda() for _ in range(2))
    sign = torch.where(torch.arange(rows) % 2 == 0, 1.0, -1.0)[:, None].cuda()
    v["x"], v["y"] = ratio * sign + dx, dy - 1.1 * ratio * sign
    if norm_y == "none":
        v["y"] = torch.zeros_like(v["y"])
    v["dn"], v["dr"] = dx + 0.5 * v["dn"], dy + 0.5 * v["dr"]
    return without(v, norm_y, norm_r)


@pytest.mark.parametrize("ratio", [100.0, 1000.0])
@pytest.mark.parametrize("norm_y,norm_r", [("none", "layer"), ("layer", "none"), ("layer", "layer")])
@pytest.mark.parametrize("rows,dim", [(4, 64), (3, 264), (4, 1928), (2, 5120), (4, 8192)])
def test_rows_far_from_zero(rows, dim, norm_y, norm_r, ratio, monkeypatch):
    v = far_inputs(rows, dim, ratio, norm_y, norm_r, rows + dim)
    step = binding.make_gated_norm(rows, dim, 0, norm_y, norm_r, EPS, FL)
    got = forward(step, v, norm_y, norm_r)
    if norm_y != "none":
        yh, eyh = again(v["y"].double(), got["stats_y"])
        u = yh * v["wy"].double() + v["by"].double()
        eu = eyh * v["wy"].double().abs() + U * (u.abs() + (yh * v["wy"].double()).abs())
        g = v["gate"].double()
        r = v["x"].double() + g * u
        close(got["r"], r, g.abs() * eu + U * (r.abs() + (g * u).abs()), "r")
    if norm_r != "none":  # (rows are fp32: r as it was stored is r as it was normed)
        check_normed(got["n"], *again(got["r"].double(), got["stats_r"]), v["wr"], v["br"], FL, "n")
    monkeypatch.setattr(ref, "again", again)
    r = got["r"] if norm_r != "none" else None
    back = backward(step, v, r, got["stats_y"], got["stats_r"], binding.make_gated_norm_workspace(step))
    # a row a team; then at most one sum of 16 places
    want = ref.backward(v["dn"], v["dr"], r, v["y"], v["gate"], v["wy"], v["by"], v["wr"], got["stats_y"], got["stats_r"],
                        norm_y, norm_r, rows, rows + 20)
    check(back, want, FL, FL)


@pytest.mark.parametrize("rows,dim", [(300, 5120), (900, 2816), (700, 512), (1300, 4096)])
def test_rows_of_16_bits_far_from_zero(rows, dim, monkeypatch):
    """Whole numbers around 192, a step of bf16 from each other: two and three rows a team."""
    v = without(inputs(rows, dim, 1, BF, FL, 8), "none", "layer")
    gen = torch.Generator().manual_seed(9)
    d = torch.randint(-3, 4, (rows, dim), generator=gen).cuda()
    v["x"], v["y"], v["dn"] = (192 + d).to(BF), torch.zeros(rows, dim, dtype=BF, device="cuda"), (v["dn"] + d).to(BF)
    step = binding.make_gated_norm(rows, dim, 0, "none", "layer", EPS, BF, FL)
    got = forward(step, v, "none", "layer")
    check_normed(got["n"], *again(got["r"].double(), got["stats_r"]), v["wr"], v["br"], BF, "n")
    monkeypatch.setattr(ref, "again", again)
    back = backward(step, v, got["r"], None, got["stats_r"], binding.make_gated_norm_workspace(step))
    want = ref.backward(v["dn"], v["dr"], got["r"], v["y"], v["gate"], None, None, v["wr"], None, got["stats_r"], "none",
                        "layer", rows, 64 + rows // 100)
    check(back, want, BF, FL)


@pytest.mark.parametrize("dtype", [BF, HF, FL])
@pytest.mark.parametrize("value", [100.0, 0.7, 0.1, 1000.3, -3.0])
@pytest.mark.parametrize("dim", [8, 256, 4096])
def test_constant_rows_of_any_value(dim, value, dtype):
    """No deviation, and a mean that is exact (dim is a power of two, the value has 11 bits): the norm is its bias."""
    value = float(torch.tensor(value, dtype=BF if dtype == FL and value < 1 else dtype if dtype != FL else HF))
    step = binding.make_gated_norm(5, dim, 0, "layer", "layer", EPS, dtype)
    x, y = (torch.full((5, dim), c, dtype=dtype, device="cuda") for c in (value, -3 * value if dtype == FL else -value))
    w, b = (torch.randn(dim, generator=torch.Generator().manual_seed(i)).to(dtype).cuda() for i in (1, 2))
    r, n = torch.empty_like(x), torch.empty_like(x)
    sy, sr = torch.empty(5, 2, device="cuda"), torch.empty(5, 2, device="cuda")
    binding.sparsp_gated_norm_fwd(step, x, y, None, w, None, w, b, r, n, sy, sr)
    assert bool((sy[:, 0] == float(y[0, 0])).all()) and bool((sr[:, 0] == value).all())
    assert torch.equal(r, x) and torch.equal(n, b.expand(5, dim))
