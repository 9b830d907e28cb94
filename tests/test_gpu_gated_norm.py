"""The residual step with its norms and gate against the plain 64-bit form; bounds are derived in step_reference.py."""
import pytest
import torch

import step_reference as ref
from layer_reference import TINY, UNIT, close
from paper_2609_32197_b200 import binding

pytestmark = pytest.mark.gpu
EPS = 1e-5
BF, HF, FL = torch.bfloat16, torch.float16, torch.float32
NAN = float("nan")


def rounded(value, error, dtype):
    return error + UNIT[dtype] * (value.abs() + error) + TINY[dtype]


def inputs(rows, dim, groups, dtype, wtype, seed=0):
    gen = torch.Generator().manual_seed(seed)

    def rand(*dims, scale=1.0, at=0.0, t=dtype):
        return (at + scale * torch.randn(*dims, generator=gen)).to(t).cuda()

    size = (1 + 3 * torch.rand(dim, generator=gen)).cuda()
    return {"x": (rand(rows, dim).float() * size + 0.5).to(dtype), "y": rand(rows, dim, scale=0.7, at=0.1),
            "gate": rand(groups, dim, scale=0.5, t=wtype), "wy": rand(dim, scale=0.3, at=1.0, t=wtype),
            "by": rand(dim, scale=0.3, t=wtype), "wr": rand(groups, dim, scale=0.3, at=1.0, t=wtype),
            "br": rand(groups, dim, scale=0.3, t=wtype), "dn": rand(rows, dim), "dr": rand(rows, dim)}


def without(v, norm_y, norm_r):
    v = dict(v)
    if norm_y == "none":
        v["wy"] = v["by"] = None
    if norm_r == "none":
        v["wr"] = v["br"] = v["dn"] = None
    return v


def forward(step, v, norm_y, norm_r, stats=True):
    rows = v["x"].shape[0]
    out = {"r": torch.full_like(v["x"], NAN), "n": torch.full_like(v["x"], NAN) if norm_r != "none" else None}
    for k, kind in (("stats_y", norm_y), ("stats_r", norm_r)):
        out[k] = torch.full((rows, 2), NAN, device="cuda") if stats and kind != "none" else None
    binding.sparsp_gated_norm_fwd(step, v["x"], v["y"], v["gate"], v["wy"], v["by"], v["wr"], v["br"], out["r"], out["n"],
                                  out["stats_y"], out["stats_r"])
    return out


def backward(step, v, r, stats_y, stats_r, ws, dx=None):
    out = {"dx": torch.full_like(v["y"], NAN) if dx is None else dx, "dy": torch.full_like(v["y"], NAN)}
    for k in ("gate", "wy", "by", "wr", "br"):
        out["d" + k] = torch.full_like(v[k], NAN) if v[k] is not None else None
    binding.sparsp_gated_norm_bwd(step, v["dn"], v["dr"], r, v["y"], v["gate"], v["wy"], v["by"], v["wr"], stats_y, stats_r,
                                  out["dx"], out["dy"], out["dgate"], out["dwy"], out["dby"], out["dwr"], out["dbr"], ws)
    return out


def check(got, want, dtype, wtype):
    for k, (value, error) in want.items():
        if got.get(k) is None:
            continue
        t = FL if k.startswith("stats") else wtype if k in ("dgate", "dwy", "dby", "dwr", "dbr") else dtype
        close(got[k][:value.shape[0]], value, rounded(value, error, t), k)
        assert bool(got[k][value.shape[0]:].isnan().all()), k  # groups without rows are left as they were


SHAPES = [
    # rows, dim, groups, dtype, weights
    (1, 8, 1, BF, BF), (1, 8, 1, FL, FL), (5, 16, 5, HF, FL), (3, 40, 1, BF, FL), (65, 128, 1, BF, BF), (33, 264, 1, FL, FL),
    (40, 512, 4, BF, FL), (12, 520, 3, HF, FL), (7, 1000, 1, FL, FL), (9, 1928, 3, FL, FL), (5, 2056, 1, HF, HF),
    (11, 4096, 1, BF, BF), (3, 5120, 3, BF, FL), (4, 8192, 1, FL, FL), (3, 8192, 1, BF, BF), (700, 640, 7, BF, BF),
    (1301, 1032, 1, BF, FL), (5000, 24, 5000, FL, FL), (9000, 136, 9, HF, FL), (2500, 32, 700, BF, FL), (1000, 5120, 3, BF, FL),
    (700, 1280, 350, HF, HF), (2000, 2560, 2, FL, FL),
]
KINDS = [("none", "layer"), ("rms", "rms"), ("layer", "none"), ("layer", "layer"), ("none", "none"), ("none", "rms")]


@pytest.mark.parametrize("norm_y,norm_r", KINDS)
@pytest.mark.parametrize("rows,dim,groups,dtype,wtype", SHAPES)
def test_forward_and_backward(rows, dim, groups, dtype, wtype, norm_y, norm_r):
    per = -(-rows // groups)
    v = without(inputs(rows, dim, groups, dtype, wtype), norm_y, norm_r)
    step = binding.make_gated_norm(rows, dim, per, norm_y, norm_r, EPS, dtype, wtype)
    got = forward(step, v, norm_y, norm_r)
    check(got, ref.forward(v["x"], v["y"], v["gate"], v["wy"], v["by"], v["wr"], v["br"], norm_y, norm_r, EPS, per), dtype, wtype)
    again = forward(step, v, norm_y, norm_r, stats=False)
    assert torch.equal(again["r"], got["r"]) and (norm_r == "none" or torch.equal(again["n"], got["n"]))

    ws = binding.make_gated_norm_workspace(step)
    ws[256:].fill_(255)  # NaN in every slot
    r = got["r"] if norm_r != "none" else None
    back = backward(step, v, r, got["stats_y"], got["stats_r"], ws)
    chain = 64 + rows // 100
    want = ref.backward(v["dn"], v["dr"], r, v["y"], v["gate"], v["wy"], v["by"], v["wr"], got["stats_y"], got["stats_r"],
                        norm_y, norm_r, per, chain)
    check(back, want, dtype, wtype)
    # the same again, in place of dr: the same bits
    dx = v["dr"].clone()
    second = backward(step, dict(v, dr=dx), r, got["stats_y"], got["stats_r"], ws, dx)
    for k in back:
        assert back[k] is None or torch.equal(second[k].nan_to_num(7.0), back[k].nan_to_num(7.0)), k


@pytest.mark.parametrize("norm_y,norm_r", [("none", "layer"), ("rms", "layer")])
def test_absent_weights_and_unwanted_gradients(norm_y, norm_r):
    rows, dim = 77, 648
    v = inputs(rows, dim, 1, BF, FL, 3)
    for k in ("gate", "wy", "by", "wr", "br"):
        v[k] = None
    step = binding.make_gated_norm(rows, dim, 0, norm_y, norm_r, EPS, BF, FL)
    got = forward(step, v, norm_y, norm_r)
    check(got, ref.forward(v["x"], v["y"], None, None, None, None, None, norm_y, norm_r, EPS, rows), BF, FL)
    ws = binding.make_gated_norm_workspace(step)
    want = ref.backward(v["dn"], None, got["r"], v["y"], None, None, None, None, got["stats_y"], got["stats_r"], norm_y, norm_r,
                        rows, 80)
    full = {"dx": torch.empty_like(v["x"]), "dy": torch.empty_like(v["x"]), "dgate": torch.empty(1, dim, device="cuda"),
            "dwy": torch.empty(dim, device="cuda") if norm_y != "none" else None, "dbr": torch.empty(1, dim, device="cuda")}

    def run(**o):
        binding.sparsp_gated_norm_bwd(step, v["dn"], None, got["r"], v["y"], None, None, None, None, got["stats_y"],
                                      got["stats_r"], o.get("dx"), o.get("dy"), o.get("dgate"), o.get("dwy"), None, None,
                                      o.get("dbr"), ws)

    run(**full)
    check(full, want, BF, FL)
    for k in full:  # each alone gives the same bits
        if full[k] is not None:
            one = torch.full_like(full[k], NAN)
            run(**{k: one})
            assert torch.equal(one, full[k]), k
    run()


def test_strides_and_in_place():
    rows, dim = 50, 264
    v = without(inputs(rows, dim, 1, BF, BF, 4), "none", "layer")
    plain = binding.make_gated_norm(rows, dim, 0, "none", "layer", EPS)
    want = forward(plain, v, "none", "layer")
    wide = {k: torch.full((rows, dim + pad), 9.0, dtype=BF, device="cuda") for k, pad in (("x", 8), ("y", 24), ("n", 24))}
    wide["x"][:, :dim], wide["y"][:, :dim] = v["x"], v["y"]
    step = binding.make_gated_norm(rows, dim, 0, "none", "layer", EPS, stride_x=dim + 8, stride_y=dim + 24, stride_n=dim + 24)
    binding.sparsp_gated_norm_fwd(step, wide["x"], wide["y"], v["gate"], None, None, v["wr"], v["br"], wide["x"], wide["y"], None, None)
    assert torch.equal(wide["x"][:, :dim], want["r"]) and torch.equal(wide["y"][:, :dim], want["n"])
    assert bool((wide["x"][:, dim:] == 9).all()) and bool((wide["y"][:, dim:] == 9).all())


def test_rows_do_not_meet():
    """Infinities and NaN of one row stay in it, and in the columns of its group."""
    rows, dim = 64, 1032
    v = inputs(rows, dim, 4, BF, FL, 5)
    step = binding.make_gated_norm(rows, dim, 16, "rms", "layer", EPS, BF, FL)
    clean = forward(step, v, "rms", "layer")
    v["x"][17, 5], v["y"][40, 1000] = float("inf"), NAN
    got = forward(step, v, "rms", "layer")
    keep = torch.ones(rows, dtype=torch.bool, device="cuda")
    keep[17] = keep[40] = False
    for k in got:
        assert torch.equal(got[k][keep], clean[k][keep]), k
    assert bool(got["n"][17].isnan().all()) and bool(got["n"][40].isnan().all())
    back = backward(step, v, got["r"], got["stats_y"], got["stats_r"], binding.make_gated_norm_workspace(step))
    assert torch.equal(back["dx"].isnan().any(1), ~keep)
    bad = back["dwr"].isnan().any(1)
    assert bad.tolist() == [False, True, True, False]


def test_constant_rows():
    """No deviation: the norm is its bias, and rstd is 1 / sqrt(eps)."""
    step = binding.make_gated_norm(3, 256, 0, "layer", "layer", EPS, FL, FL)
    x, y = torch.full((3, 256), 3.0, device="cuda"), torch.full((3, 256), -2.0, device="cuda")
    b = torch.randn(256, device="cuda")
    r, n, sy, sr = torch.empty_like(x), torch.empty_like(x), torch.empty(3, 2, device="cuda"), torch.empty(3, 2, device="cuda")
    binding.sparsp_gated_norm_fwd(step, x, y, None, None, None, None, b, r, n, sy, sr)
    assert torch.equal(r, x) and torch.equal(n, b.expand(3, 256))
    assert torch.allclose(sy, torch.tensor([-2.0, EPS ** -0.5], device="cuda").expand(3, 2), rtol=1e-6)


def test_gradients_against_differences():
    """The backward pass against differences of the forward pass, both in fp32: 64-bit differences of the plain form would
    test that form alone."""
    rows, dim, h = 6, 64, 2.0 ** -6
    v = inputs(rows, dim, 2, FL, FL, 7)
    step = binding.make_gated_norm(rows, dim, 3, "layer", "rms", EPS, FL, FL)
    got = forward(step, v, "layer", "rms")
    back = backward(step, v, got["r"], got["stats_y"], got["stats_r"], binding.make_gated_norm_workspace(step))

    def loss(w):
        o = forward(step, w, "layer", "rms")
        return float((o["r"].double() * v["dr"].double()).sum() + (o["n"].double() * v["dn"].double()).sum())

    gen = torch.Generator().manual_seed(8)
    for k in ("x", "y", "gate", "wy", "by", "wr", "br"):
        d = torch.randn(v[k].shape, generator=gen).cuda()
        diff = (loss(dict(v, **{k: v[k] + h * d})) - loss(dict(v, **{k: v[k] - h * d}))) / (2 * h)
        mine = float((back["d" + k].double() * d.double()).sum())
        # third derivatives times h^2 / 6, and the values' own roundings over 2 h: both under a thousandth of the terms' norm
        size = float((back["d" + k].double() * d.double()).norm()) + float(v["dr"].norm()) + float(v["dn"].norm())
        assert abs(diff - mine) <= 2e-3 * size, (k, diff, mine)


def test_no_rows():
    step = binding.make_gated_norm(0, 64, 0, "rms", "layer", EPS, BF, FL)
    binding.sparsp_gated_norm_fwd(step, *[None] * 11)
    dwy, dby = torch.full((64,), NAN, device="cuda"), torch.full((64,), NAN, device="cuda")
    ws = binding.make_gated_norm_workspace(step)
    binding.sparsp_gated_norm_bwd(step, *[None] * 13, dwy, dby, None, None, ws)
    assert bool((dwy == 0).all()) and bool((dby == 0).all())
