"""Plain 64-bit forms of the token-wise operators, written from their formulas, for the tests."""
import math

import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}  # half a step, relative
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}  # half a step near zero
F32 = 2.0 ** -24


def rotate(x, cos, sin, rotated, rot_begin, half, inverse):
    """x [B][H][N][d] in 64 bits; cos, sin [B][N][pairs]; rotated [B][N]."""
    r = cos.shape[-1]
    first = [rot_begin + i if half else rot_begin + 2 * i for i in range(r)]
    second = [rot_begin + r + i if half else rot_begin + 2 * i + 1 for i in range(r)]
    sin = -sin if inverse else sin
    y = x.clone()
    c, s = cos[:, None], sin[:, None]
    a, b = x[..., first], x[..., second]
    on = rotated[:, None, :, None]
    y[..., first] = torch.where(on, a * c - b * s, a)
    y[..., second] = torch.where(on, a * s + b * c, b)
    return y


def layer_norm(x, w, b, eps, per_group):
    """x [R][D] in 64 bits; w, b [G][D] or None -> y, mean, rstd"""
    mean = x.mean(1)
    d = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((d * d).mean(1) + eps)
    y = d * rstd[:, None]
    g = torch.arange(x.shape[0], device=x.device) // per_group
    if w is not None:
        y = y * w[g]
    if b is not None:
        y = y + b[g]
    return y, mean, rstd


def layer_norm_back(dy, x, w, mean, rstd, per_group, groups):
    g = torch.arange(x.shape[0], device=x.device) // per_group
    xh = (x - mean[:, None]) * rstd[:, None]
    a = dy if w is None else dy * w[g]
    D = x.shape[1]
    dx = rstd[:, None] * (a - a.sum(1, keepdim=True) / D - xh * (a * xh).sum(1, keepdim=True) / D)
    dw = torch.zeros(groups, D, dtype=x.dtype, device=x.device).index_add_(0, g, dy * xh)
    db = torch.zeros(groups, D, dtype=x.dtype, device=x.device).index_add_(0, g, dy)
    return dx, dw, db


def activation(kind, x):
    """a(x), a'(x)"""
    if kind == "silu":
        s = 1 / (1 + torch.exp(-x))
        return x * s, s + x * s * (1 - s)
    if kind == "gelu_tanh":
        k = math.sqrt(2 / math.pi)
        t = torch.tanh(k * (x + 0.044715 * x ** 3))
        return x / 2 * (1 + t), (1 + t) / 2 + x / 2 * (1 - t * t) * k * (1 + 3 * 0.044715 * x * x)
    c = (1 + torch.erf(x / math.sqrt(2))) / 2
    return x * c, c + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)


def close(got, want, bound, what):
    """|got - want| <= bound element by element; NaN and infinities in the same places."""
    got, want = got.double(), want.double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN elsewhere"
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), f"{what}: infinities elsewhere"
    over = ((got - want).abs() - bound)[fine]
    if over.numel():
        at = int(over.argmax())
        assert over[at] <= 0, f"{what}: off by {float((got - want).abs()[fine][at])}, bound {float(bound.expand_as(want)[fine][at])}"
