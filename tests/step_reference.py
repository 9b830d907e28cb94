"""The residual step in plain 64-bit form, each result with how far an fp32 computation of it may be off.

u = 2^-24.  A sum of D terms over a tree of depth log2 D after at most 40 terms a thread is off by at most 50 u of the sum
of its terms' magnitudes; a product or a sum of two by u of its result; errors of what goes in are carried along to
first order, with 1 % on top for the rest."""
import torch

from layer_reference import F32 as U

MORE = 1.01


def rows_of(w, g, like):
    """A weight for each row; None: ones."""
    return torch.ones_like(like) if w is None else w.double()[g]


def normed(kind, v, ev, eps):
    """v [R][D], off by ev -> (vh, its error, mean, its error, rstd, its error)"""
    top = v.abs().amax(1, keepdim=True)
    if kind == "layer":
        mean, em = v.mean(1, keepdim=True), ev.mean(1, keepdim=True) + 51 * U * v.abs().mean(1, keepdim=True)
    else:
        mean = em = torch.zeros_like(top)
    d, ed = v - mean, ev + em + U * (v.abs() + mean.abs())
    q = (d * d).mean(1, keepdim=True)
    eq = (2 * d.abs() * ed + ed * ed).mean(1, keepdim=True) + 53 * U * q
    rstd = 1 / torch.sqrt(q + eps)
    er = rstd * (eq / (2 * (q + eps)) + 5 * U) * MORE
    vh = d * rstd
    return vh, (ed * rstd + d.abs() * er + 2 * U * vh.abs()) * MORE, mean, em, rstd, er


def forward(x, y, gate, wy, by, wr, br, norm_y, norm_r, eps, per):
    """-> {name: (value, error)}; stats [R][2]"""
    x, y = x.double(), y.double()
    g = torch.arange(x.shape[0], device=x.device) // per
    out, u, eu = {}, y, torch.zeros_like(y)
    if norm_y != "none":
        yh, eyh, m, em, r, er = normed(norm_y, y, eu, eps)
        out["stats_y"] = torch.cat((m, r), 1), torch.cat((em, er), 1)
        w = torch.ones_like(yh) if wy is None else wy.double().expand_as(yh)
        b = torch.zeros_like(yh) if by is None else by.double().expand_as(yh)
        u = yh * w + b
        eu = eyh * w.abs() + U * (u.abs() + (yh * w).abs())
    gate = rows_of(gate, g, u)
    r = x + gate * u
    er = (gate.abs() * eu + U * (r.abs() + (gate * u).abs())) * MORE
    out["r"] = r, er
    if norm_r != "none":
        rh, erh, m, em, rs, ers = normed(norm_r, r, er, eps)
        out["stats_r"] = torch.cat((m, rs), 1), torch.cat((em, ers), 1)
        w, b = rows_of(wr, g, rh), torch.zeros_like(rh) if br is None else br.double()[g]
        n = rh * w + b
        out["n"] = n, erh * w.abs() + U * (n.abs() + (rh * w).abs())
    return out


def again(v, stats):
    """v normed by its kept statistics, and the error"""
    m, r = stats.double()[:, :1], stats.double()[:, 1:]
    vh = (v - m) * r
    return vh, 3 * U * (vh.abs() + (v.abs() + m.abs()) * r)


def through(kind, a, ea, vh, evh, stats):
    """The gradient of what a norm took, and the error."""
    r = stats.double()[:, 1:]
    m1 = (a * vh).mean(1, keepdim=True)
    e1 = (a.abs() * evh + ea * vh.abs() + 55 * U * (a * vh).abs()).mean(1, keepdim=True)
    m0, e0 = torch.zeros_like(m1), torch.zeros_like(m1)
    if kind == "layer":
        m0, e0 = a.mean(1, keepdim=True), (ea + 52 * U * a.abs()).mean(1, keepdim=True)
    back = r * (a - m0 - vh * m1)
    size = a.abs() + m0.abs() + (vh * m1).abs()
    return back, r * (ea + e0 + vh.abs() * e1 + evh * m1.abs() + 5 * U * size) * MORE


def backward(dn, dr, r, y, gate, wy, by, wr, stats_y, stats_r, norm_y, norm_r, per, chain):
    """-> {name: (value, error)}.  chain: the longest run of additions one after the other in a column's sum."""
    y = y.double()
    R, D = y.shape
    g = torch.arange(R, device=y.device) // per
    groups = -(-R // per)
    out = {}

    def column(terms, errors):
        s, e = (torch.zeros(groups, D, dtype=torch.float64, device=y.device).index_add_(0, g, v)
                for v in (terms, errors + chain * U * terms.abs()))
        return s, e * MORE

    t, et = (torch.zeros_like(y) if dr is None else dr.double()), torch.zeros_like(y)
    if norm_r != "none":
        dn, r = dn.double(), r.double()
        rh, erh = again(r, stats_r)
        a = dn * rows_of(wr, g, dn)
        back, eb = through(norm_r, a, U * a.abs(), rh, erh, stats_r)
        out["dwr"], out["dbr"] = column(dn * rh, dn.abs() * erh), column(dn, torch.zeros_like(dn))
        et = eb + 2 * U * (t.abs() + back.abs())
        t = t + back
    out["dx"] = t, et
    gate_rows = rows_of(gate, g, t)
    if norm_y == "none":
        out["dy"] = t * gate_rows, et * gate_rows.abs() + U * (t * gate_rows).abs()
        out["dgate"] = column(t * y, et * y.abs())
        return out
    yh, eyh = again(y, stats_y)
    w = torch.ones(D, dtype=torch.float64, device=y.device) if wy is None else wy.double()
    b = torch.zeros_like(w) if by is None else by.double()
    p = t * gate_rows * w
    out["dy"] = through(norm_y, p, et * (gate_rows * w).abs() + 3 * U * p.abs(), yh, eyh, stats_y)
    c, ec = column(t * yh, et * yh.abs() + t.abs() * eyh)
    d, ed = column(t, et)
    out["dgate"] = w * c + b * d, w.abs() * ec + b.abs() * ed + 3 * U * ((w * c).abs() + (b * d).abs())
    G = torch.ones(groups, D, dtype=torch.float64, device=y.device) if gate is None else gate.double()[:groups]
    for k, (s, e) in (("dwy", (c, ec)), ("dby", (d, ed))):
        size = (G * s).abs().sum(0)
        out[k] = (G * s).sum(0), (G.abs() * e).sum(0) + (groups + chain) * U * size
    return out
