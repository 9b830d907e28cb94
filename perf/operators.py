"""The work that the token-wise operators beside the attention are judged by: rotary positions on Q and K, layer norm and
the gated feed-forward half of a layer, each in every direction that a user calls it in.

A case is a dict of plain values.  `op` says which call one pass makes:

  rotary     Q and K (or Q alone) rotated by the positions of their tokens, or rotated back (the gradient)
  norm_fwd   layer norm with the row statistics that training keeps, or without
  norm_bwd   its gradients: dx, and the weight's and bias' summed over the rows of each group
  ffn_fwd    act(X Wg^T) * (X Wu^T), or the same with both projections kept for the backward pass
  ffn_bwd    dX, dWg and dWu from dH and the kept projections

`own` chooses between the plain form (elementary torch operations in 32 bits, rounded once) and the library's calls.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}


def _rotary(name, heads, head_dim, grid, pairs, *, n_text=0, batch=1, layout="HND", pairing="interleaved", rot_begin=0,
            dtype="bf16", inverse=False, both=True, table=0, scaling="none", factor=1.0):
    return {"name": name, "op": "rotary", "heads": heads, "head_dim": head_dim, "grid_t": grid[0], "grid_h": grid[1],
            "grid_w": grid[2], "pairs_t": pairs[0], "pairs_h": pairs[1], "pairs_w": pairs[2], "n_text": n_text,
            "batch": batch, "layout": layout, "pairing": pairing, "rot_begin": rot_begin, "dtype": dtype,
            "inverse": inverse, "both": both, "table": table, "scaling": scaling, "factor": factor}


def _norm(name, op, rows, dim, *, groups=1, dtype="bf16", weights="bf16", stats=True):
    return {"name": name, "op": op, "rows": rows, "dim": dim, "groups": groups, "dtype": dtype, "weights": weights,
            "stats": stats}


def _ffn(name, op, tokens, dim, hidden, *, dtype="bf16", activation="silu", keep=False):
    return {"name": name, "op": op, "tokens": tokens, "dim": dim, "hidden": hidden, "dtype": dtype,
            "activation": activation, "keep": keep}


def listed():
    return [
        # Q and K of a long video layer on its latent grid: 40 heads of 128, the channel pairs shared out among t, h and w
        _rotary("rotary-wan", 40, 128, (21, 45, 80), (22, 21, 21)),
        # the gradient of a head_dim-64 layer with text behind the video, token-major, pairs half a head apart, part of the head
        _rotary("rotary-cog-back", 48, 64, (13, 30, 45), (8, 8, 8), n_text=226, layout="NHD", pairing="half", dtype="fp16",
                inverse=True),
        # one new token of each of 64 requests, at positions of their own in a context four times the original length
        _rotary("rotary-token", 32, 128, (1, 1, 1), (32, 0, 0), batch=64, layout="NHD", pairing="half", table=131072,
                scaling="yarn", factor=4.0),
        # the smallest layer in use: latency
        _norm("norm-tiny", "norm_fwd", 4096, 128, stats=False),
        # a long video layer's norm, as training calls it
        _norm("norm-wan", "norm_fwd", 75600, 5120, weights="fp32"),
        # its backward pass
        _norm("norm-wan-back", "norm_bwd", 75600, 5120),
        # two sequences with weights of their own (a norm modulated by each sequence's condition), odd width, 32 bits
        _norm("norm-odd-back", "norm_bwd", 2 * 7777, 1921, groups=2, dtype="fp32", weights="fp32"),
        # a single token: every weight is read for it
        _ffn("ffn-token", "ffn_fwd", 1, 5120, 13824),
        # the text tokens of one prompt
        _ffn("ffn-text", "ffn_fwd", 226, 1920, 7680, dtype="fp16", activation="gelu_tanh"),
        # half of a long video layer's tokens, both projections kept for training
        _ffn("ffn-train", "ffn_fwd", 37800, 5120, 13824, keep=True),
        # its backward pass: the largest case
        _ffn("ffn-train-back", "ffn_bwd", 37800, 5120, 13824),
        # a small odd-sized layer's backward pass
        _ffn("ffn-odd-back", "ffn_bwd", 1003, 1160, 2504, activation="gelu"),
    ]


def _log_int(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(("rotary", "norm_fwd", "norm_bwd", "ffn_fwd", "ffn_fwd", "ffn_bwd"))
    dtype = rng.choice(("bf16", "bf16", "fp16", "fp32"))
    if op == "rotary":
        head_dim, heads = rng.choice((64, 128)), rng.randint(1, 40)
        tokens = _log_int(rng, 1, 75600)
        if rng.random() < 0.5:  # a latent grid
            t = rng.randint(1, min(21, tokens))
            h = _log_int(rng, 1, max(1, min(60, tokens // t)))
            grid, n_text, batch, table = (t, h, max(1, min(100, tokens // (t * h)))), rng.choice((0, 0, rng.randint(1, 300))), 1, 0
            p = head_dim // 8
            pairs = rng.choice(((head_dim // 2 - 2 * p, p, p), (p, p, p), (head_dim // 2 - 2 * (p + 1), p + 1, p + 1)))
        else:  # text alone, any position in a table
            batch = _log_int(rng, 1, 64)
            grid, n_text = (max(1, tokens // batch), 1, 1), 0
            table, pairs = max(grid[0], rng.choice((8192, 131072))), (rng.choice((head_dim // 2, head_dim // 4)), 0, 0)
        rot_begin = rng.choice((0, head_dim - 2 * sum(pairs)))
        scaling = rng.choice(("none", "linear", "ntk", "yarn"))
        return _rotary("", heads, head_dim, grid, pairs, n_text=n_text, batch=batch, layout=rng.choice(("HND", "NHD")),
                       pairing=rng.choice(("interleaved", "half")), rot_begin=rot_begin, dtype=dtype,
                       inverse=rng.random() < 0.4, both=rng.random() < 0.7, table=table, scaling=scaling,
                       factor=1.0 if scaling == "none" else rng.choice((2.0, 4.0, 8.0)))
    if op.startswith("norm"):
        dim = _log_int(rng, 16, 8192)
        if rng.random() < 0.6:
            dim = (dim + 7) // 8 * 8
        groups = rng.choice((1, 1, 2, 5))
        per_group = _log_int(rng, 1, max(1, min(75600, 75600 * 5120 // dim // (2 if dtype == "fp32" else 1)) // groups))
        return _norm("", op, groups * per_group, dim, groups=groups, dtype=dtype, weights=rng.choice((dtype, "fp32")),
                     stats=op == "norm_bwd" or rng.random() < 0.6)
    dtype = "bf16" if dtype == "fp32" else dtype
    dim, hidden = _log_int(rng, 8, 640) * 8, _log_int(rng, 16, 1728) * 8
    tokens = _log_int(rng, 1, 37800 if op == "ffn_bwd" else 75600)
    return _ffn("", op, tokens, dim, hidden, dtype=dtype, activation=rng.choice(("silu", "gelu_tanh", "gelu")),
                keep=op == "ffn_fwd" and rng.random() < 0.5)


# ---- inputs ---------------------------------------------------------------------------------------------------------


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(gen, shape, dtype, scale=1.0):
    out = torch.empty(shape, dtype=dtype, device="cuda")
    return out.normal_(0.0, scale, generator=gen)


def _n_tokens(c):
    return c["grid_t"] * c["grid_h"] * c["grid_w"] + c["n_text"]


def _frequencies(c):
    """Radians per position of every pair, one tensor in 64 bits per coordinate, and the amplitude of cos and sin."""
    found, s = [], c["factor"]
    amplitude = 0.1 * math.log(s) + 1.0 if c["scaling"] == "yarn" else 1.0
    for n in (c["pairs_t"], c["pairs_h"], c["pairs_w"]):
        i = torch.arange(n, dtype=torch.float64)
        theta = 10000.0 * s ** (n / (n - 1)) if c["scaling"] == "ntk" and n > 1 else 10000.0
        f = theta ** (-i / max(n, 1))
        if c["scaling"] == "linear":
            f = f / s
        if c["scaling"] == "yarn":
            # by the turns that a pair makes over the original context: over 32 it stays, under 1 it is stretched
            at = lambda b: n * math.log(4096 / (2 * math.pi * b)) / math.log(10000.0)  # noqa: E731  the pair that turns b times
            low, high = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), n - 1)
            stay = 1.0 - ((i - low) / max(high - low, 0.001)).clamp(0.0, 1.0)
            f = f * stay + f / s * (1.0 - stay)
        found.append(f)
    return found, amplitude


def _lengths(c):
    return (c["table"] or c["grid_t"], c["grid_h"], c["grid_w"])


def _grid_positions(c):
    """[tokens][3], -1 for text tokens."""
    t, h, w = torch.meshgrid(*(torch.arange(c[k], dtype=torch.int32, device="cuda") for k in ("grid_t", "grid_h", "grid_w")),
                             indexing="ij")
    video = torch.stack((t.reshape(-1), h.reshape(-1), w.reshape(-1)), 1)
    return torch.cat((video, torch.full((c["n_text"], 3), -1, dtype=torch.int32, device="cuda")))


def _inputs(c, seed):
    gen = _generator(seed)
    dt = DTYPES[c["dtype"]]
    if c["op"] == "rotary":
        n = _n_tokens(c)
        dims = (c["batch"], c["heads"], n, c["head_dim"]) if c["layout"] == "HND" else (c["batch"], n, c["heads"], c["head_dim"])
        x = {"q": _normal(gen, dims, dt)}
        if c["both"]:
            x["k"] = _normal(gen, dims, dt)
        if c["table"]:  # every request begins at a place of its own
            first = torch.randint(0, c["table"] - c["grid_t"] + 1, (c["batch"], 1), generator=gen, device="cuda", dtype=torch.int32)
            x["positions"] = torch.zeros((c["batch"], n, 3), dtype=torch.int32, device="cuda")
            x["positions"][:, :, 0] = first + torch.arange(n, dtype=torch.int32, device="cuda")
        return x
    if c["op"].startswith("norm"):
        rows, dim, wt = c["rows"], c["dim"], DTYPES[c["weights"]]
        # hidden states: channels of different sizes, a few of them far larger than the rest, and a mean of their own
        size = torch.empty(dim, device="cuda").normal_(0.0, 0.5, generator=gen).exp_()
        size[torch.randint(0, dim, (max(1, dim // 256),), generator=gen, device="cuda")] *= 8.0
        x = {"x": _normal(gen, (rows, dim), dt).mul_(size.to(dt)).add_(0.5)}
        x["w"] = _normal(gen, (c["groups"], dim), torch.float32, 0.2).add_(1.0).to(wt)
        x["b"] = _normal(gen, (c["groups"], dim), wt, 0.2)
        if c["op"] == "norm_bwd":
            x["dy"] = _normal(gen, (rows, dim), dt)
            x["mean"], x["rstd"] = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
            step = max(1, (1 << 27) // dim)
            for r in range(0, rows, step):
                part = x["x"][r:r + step].double()
                x["mean"][r:r + step] = part.mean(1)
                x["rstd"][r:r + step] = (part.var(1, unbiased=False) + EPS).rsqrt()
        return x
    m, d, f = c["tokens"], c["dim"], c["hidden"]
    x = {"x": _normal(gen, (m, d), dt), "wg": _normal(gen, (f, d), dt, d ** -0.5), "wu": _normal(gen, (f, d), dt, d ** -0.5)}
    if c["op"] == "ffn_bwd":
        x["gate"], x["up"] = x["x"] @ x["wg"].T, x["x"] @ x["wu"].T
        x["dh"] = _normal(gen, (m, f), dt)
    return x


EPS = 1e-5


def prepare(case, seed):
    c = dict(case)
    x = _inputs(c, seed)
    if c["op"] == "rotary":
        freq, amplitude = _frequencies(c)
        if not own:  # the table that a program keeps: (cos, sin) of every position of every coordinate
            x["table"] = []
            for f, length in zip(freq, _lengths(c)):
                angle = torch.arange(length, dtype=torch.float64, device="cuda")[:, None] * f.cuda()
                x["table"].append(((angle.cos() * amplitude).float(), (angle.sin() * amplitude).float()))
            if not c["table"]:
                x["positions"] = _grid_positions(c)
    if own:
        _plan(c, x)
    return c, x


def _plan(c, x):
    """What a program of the library keeps beside its data: descriptions, tables, buffers for results, a workspace."""
    from paper_2609_32197_b200 import binding

    dt = DTYPES[c["dtype"]]
    if c["op"] == "rotary":
        x["shape"] = binding.make_shape(c["heads"], c["head_dim"], (c["grid_t"], c["grid_h"], c["grid_w"]), c["n_text"], 64,
                                        batch=c["batch"], layout=c["layout"])
        x["rotary"] = binding.make_rotary((c["pairs_t"], c["pairs_h"], c["pairs_w"]), _lengths(c), pairing=c["pairing"],
                                          rot_begin=c["rot_begin"], dtype=dt)
        freq, amplitude = [], 1.0
        for n in (c["pairs_t"], c["pairs_h"], c["pairs_w"]):
            f, amplitude = binding.sparsp_rotary_frequencies(n, 10000.0, c["scaling"], c["factor"], 4096)
            freq.append(f)
        x["table"] = binding.make_rotary_table(x["rotary"], torch.cat(freq), amplitude)
        x["out"] = {k: torch.empty_like(x[k]) for k in ("q", "k") if k in x}
        x["workspace"] = binding.make_status_workspace()
    elif c["op"].startswith("norm"):
        x["norm"] = binding.make_norm(c["rows"], c["dim"], rows_per_group=c["rows"] // c["groups"], eps=EPS, dtype=dt,
                                      weight_dtype=DTYPES[c["weights"]])
        if c["op"] == "norm_fwd":
            x["out"] = {"y": torch.empty_like(x["x"])}
            if c["stats"]:
                x["out"]["mean"], x["out"]["rstd"] = (torch.empty(c["rows"], device="cuda") for _ in range(2))
        else:
            x["out"] = {"dx": torch.empty_like(x["x"]), "dw": torch.empty_like(x["w"]), "db": torch.empty_like(x["b"])}
            x["workspace"] = binding.make_norm_workspace(x["norm"])
    else:
        x["ffn"] = binding.make_ffn(c["tokens"], c["dim"], c["hidden"], activation=c["activation"], dtype=dt)
        x["workspace"] = binding.make_ffn_workspace(x["ffn"], backward=c["op"] == "ffn_bwd")
        if c["op"] == "ffn_fwd":
            x["out"] = {k: torch.empty((c["tokens"], c["hidden"]), dtype=dt, device="cuda")
                        for k in (("h", "gate", "up") if c["keep"] else ("h",))}
        else:
            x["out"] = {"dx": torch.empty_like(x["x"]), "dwg": torch.empty_like(x["wg"]), "dwu": torch.empty_like(x["wu"])}


# ---- one pass -------------------------------------------------------------------------------------------------------


def run(state):
    c, x = state
    if own:
        return _run_own(c, x)
    return {"rotary": _plain_rotary, "norm_fwd": _plain_norm_fwd, "norm_bwd": _plain_norm_bwd, "ffn_fwd": _plain_ffn_fwd,
            "ffn_bwd": _plain_ffn_bwd}[c["op"]](c, x)


def _run_own(c, x):
    from paper_2609_32197_b200 import binding

    o = x["out"]
    if c["op"] == "rotary":
        binding.sparsp_rotary_apply(x["shape"], x["rotary"], x["table"], x.get("positions"), (0, 0, 0), x["q"], x.get("k"),
                                    o["q"], o.get("k"), c["inverse"], x["workspace"])
    elif c["op"] == "norm_fwd":
        binding.sparsp_layer_norm_fwd(x["norm"], x["x"], x["w"], x["b"], o["y"], o.get("mean"), o.get("rstd"))
    elif c["op"] == "norm_bwd":
        binding.sparsp_layer_norm_bwd(x["norm"], x["dy"], x["x"], x["w"], x["mean"], x["rstd"], o["dx"], o["dw"], o["db"],
                                      x["workspace"])
    elif c["op"] == "ffn_fwd":
        binding.sparsp_gated_ffn_fwd(x["ffn"], x["x"], x["wg"], x["wu"], o["h"], o.get("gate"), o.get("up"), x["workspace"])
    else:
        binding.sparsp_gated_ffn_bwd(x["ffn"], x["dh"], x["x"], x["wg"], x["wu"], x["gate"], x["up"], o["dx"], o["dwg"],
                                     o["dwu"], x["workspace"])
    return o


def _plain_rotary(c, x):
    pos = x["positions"]
    rotated = pos[..., 0] >= 0
    cos, sin = ([t[k][pos[..., a].clamp(min=0).long()] for a, t in enumerate(x["table"]) if t[k].shape[1]] for k in (0, 1))
    cos, sin = torch.cat(cos, -1), torch.cat(sin, -1)
    if c["inverse"]:
        sin = -sin
    axis = -3 if c["layout"] == "HND" else -2  # the heads' place
    cos, sin, rotated = cos.unsqueeze(axis), sin.unsqueeze(axis), rotated[..., None].unsqueeze(axis)
    r, lo = c["pairs_t"] + c["pairs_h"] + c["pairs_w"], c["rot_begin"]
    out = {}
    for k in ("q", "k"):
        if k not in x:
            continue
        part = x[k][..., lo:lo + 2 * r].float()
        if c["pairing"] == "half":
            a, b = part[..., :r], part[..., r:]
            turned = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
        else:
            a, b = part[..., 0::2], part[..., 1::2]
            turned = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
        out[k] = x[k].clone()
        out[k][..., lo:lo + 2 * r] = torch.where(rotated, turned, part).to(x[k].dtype)
    return out


def _per_row(c, w):
    """A weight of each group against the rows of its group: [groups][1][dim]."""
    return w.float()[:, None, :]


def _plain_norm_fwd(c, x):
    v = x["x"].float().view(c["groups"], -1, c["dim"])
    mean = v.mean(-1, keepdim=True)
    v = v - mean
    rstd = (v.square().mean(-1, keepdim=True) + EPS).rsqrt()
    y = v * rstd * _per_row(c, x["w"]) + _per_row(c, x["b"])
    out = {"y": y.to(x["x"].dtype).view_as(x["x"])}
    if c["stats"]:
        out["mean"], out["rstd"] = mean.reshape(-1), rstd.reshape(-1)
    return out


def _plain_norm_bwd(c, x):
    v, dy = (x[k].float().view(c["groups"], -1, c["dim"]) for k in ("x", "dy"))
    mean, rstd = (x[k].view(c["groups"], -1, 1) for k in ("mean", "rstd"))
    xh = (v - mean) * rstd
    a = dy * _per_row(c, x["w"])
    dx = rstd * (a - a.mean(-1, keepdim=True) - xh * (a * xh).mean(-1, keepdim=True))
    return {"dx": dx.to(x["x"].dtype).view_as(x["x"]), "dw": (dy * xh).sum(1).to(x["w"].dtype), "db": dy.sum(1).to(x["b"].dtype)}


def _act(name, g):
    """The activation and its slope at g."""
    if name == "silu":
        s = 1 / (1 + torch.exp(-g))
        return g * s, s * (1 + g * (1 - s))
    if name == "gelu_tanh":
        k = math.sqrt(2 / math.pi)
        t = torch.tanh(k * (g + 0.044715 * g * g * g))
        return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * k * (1 + 3 * 0.044715 * g * g)
    p = 0.5 * (1 + torch.erf(g / math.sqrt(2)))
    return g * p, p + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)


def _plain_ffn_fwd(c, x):
    v = x["x"].float()
    gate, up = v @ x["wg"].float().T, v @ x["wu"].float().T
    dt = x["x"].dtype
    out = {"h": (_act(c["activation"], gate)[0] * up).to(dt)}
    if c["keep"]:
        out["gate"], out["up"] = gate.to(dt), up.to(dt)
    return out


def _plain_ffn_bwd(c, x):
    value, slope = _act(c["activation"], x["gate"].float())
    dh, dt = x["dh"].float(), x["x"].dtype
    dup = dh * value
    dgate = dh * x["up"].float() * slope
    del value, slope, dh
    v = x["x"].float()
    return {"dx": (dgate @ x["wg"].float() + dup @ x["wu"].float()).to(dt), "dwg": (dgate.T @ v).to(dt), "dwu": (dup.T @ v).to(dt)}


# ---- what a pass cannot do without ----------------------------------------------------------------------------------


def work(case):
    c = case
    e = BYTES[c["dtype"]]
    if c["op"] == "rotary":
        n, tensors = _n_tokens(c) * c["batch"], 2 if c["both"] else 1
        pairs = (c["pairs_t"], c["pairs_h"], c["pairs_w"])
        rows = n * c["heads"] * tensors
        if c["table"]:
            table = min(n, c["table"]) * pairs[0] * 8 + n * 12
        else:
            table = sum(p * q for p, q in zip(pairs, _lengths(c))) * 8
        return {"bytes": rows * c["head_dim"] * e * 2 + table, "flops": rows * sum(pairs) * 6}
    if c["op"].startswith("norm"):
        size, wsize = c["rows"] * c["dim"], c["groups"] * c["dim"] * BYTES[c["weights"]]
        if c["op"] == "norm_fwd":
            return {"bytes": 2 * size * e + 2 * wsize + (8 * c["rows"] if c["stats"] else 0), "flops": 8 * size}
        return {"bytes": 3 * size * e + 3 * wsize + 8 * c["rows"], "flops": 13 * size}
    m, d, f = c["tokens"], c["dim"], c["hidden"]
    if c["op"] == "ffn_fwd":
        return {"bytes": e * (m * d + 2 * f * d + m * f * (3 if c["keep"] else 1)), "flops": 4 * m * d * f}
    return {"bytes": e * (2 * m * d + 4 * f * d + 3 * m * f), "flops": 8 * m * d * f}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------


def exact(case, seed):
    c = dict(case)
    x = _inputs(c, seed)
    return {"rotary": _exact_rotary, "norm_fwd": _exact_norm_fwd, "norm_bwd": _exact_norm_bwd, "ffn_fwd": _exact_ffn_fwd,
            "ffn_bwd": _exact_ffn_bwd}[c["op"]](c, x)


def _exact_rotary(c, x):
    """Each pair as a complex number, multiplied by amplitude * e^(i angle)."""
    freq, amplitude = _frequencies(c)
    pos = x["positions"] if c["table"] else _grid_positions(c)
    angle = torch.cat([pos[..., a:a + 1].double() * f.cuda() for a, f in enumerate(freq)], -1)
    turn = torch.polar(torch.full_like(angle, amplitude), -angle if c["inverse"] else angle)
    turn = torch.where(pos[..., :1] >= 0, turn, torch.ones_like(turn))
    turn = turn.unsqueeze(-3 if c["layout"] == "HND" else -2)
    r, lo, out = turn.shape[-1], c["rot_begin"], {}
    for k in ("q", "k"):
        if k not in x:
            continue
        y = x[k].double()
        if c["pairing"] == "half":
            z = torch.complex(y[..., lo:lo + r], y[..., lo + r:lo + 2 * r]) * turn
            y[..., lo:lo + r], y[..., lo + r:lo + 2 * r] = z.real, z.imag
        else:
            z = torch.complex(y[..., lo:lo + 2 * r:2], y[..., lo + 1:lo + 2 * r:2]) * turn
            y[..., lo:lo + 2 * r:2], y[..., lo + 1:lo + 2 * r:2] = z.real, z.imag
        out[k] = y
        del z
    return out


def _chunks(c):
    """Rows [a, b) of one group at a time, few enough to be held in 64 bits several times over."""
    per, step = c["rows"] // c["groups"], max(1, (1 << 27) // c["dim"])
    for g in range(c["groups"]):
        for a in range(g * per, (g + 1) * per, step):
            yield g, a, min(a + step, (g + 1) * per)


def _exact_norm_fwd(c, x):
    y, stats = torch.empty(x["x"].shape, dtype=torch.float64, device="cuda"), []
    for g, a, b in _chunks(c):
        v = x["x"][a:b].double()
        var, mean = torch.var_mean(v, 1, unbiased=False, keepdim=True)
        y[a:b] = (v - mean) / torch.sqrt(var + EPS) * x["w"][g].double() + x["b"][g].double()
        stats.append((mean[:, 0], 1 / torch.sqrt(var[:, 0] + EPS)))
    out = {"y": y}
    if c["stats"]:
        out["mean"], out["rstd"] = (torch.cat(s) for s in zip(*stats))
    return out


def _exact_norm_bwd(c, x):
    dx = torch.empty(x["x"].shape, dtype=torch.float64, device="cuda")
    dw, db = (torch.zeros((c["groups"], c["dim"]), dtype=torch.float64, device="cuda") for _ in range(2))
    for g, a, b in _chunks(c):
        r = x["rstd"][a:b, None].double()
        xh, dy = (x["x"][a:b].double() - x["mean"][a:b, None].double()) * r, x["dy"][a:b].double()
        dw[g] += torch.einsum("rd,rd->d", dy, xh)
        db[g] += dy.sum(0)
        p = dy * x["w"][g].double()
        along = torch.einsum("rd,rd->r", p, xh)[:, None] / c["dim"]
        dx[a:b] = (p - p.sum(1, keepdim=True) / c["dim"] - along * xh) * r
    return {"dx": dx, "dw": dw, "db": db}


def _act64(name, g):
    """The activation in 64 bits, written so that autograd gives its slope."""
    if name == "silu":
        return g * torch.special.expit(g)
    if name == "gelu_tanh":
        return g * torch.special.expit(2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3))
    return g * torch.special.ndtr(g)


def _exact_ffn_fwd(c, x):
    v = x["x"].double()
    gate, up = torch.einsum("md,fd->mf", v, x["wg"].double()), torch.einsum("md,fd->mf", v, x["wu"].double())
    out = {"h": _act64(c["activation"], gate).mul_(up)}
    if c["keep"]:
        out["gate"], out["up"] = gate, up
    return out


def _exact_ffn_bwd(c, x):
    m = c["tokens"]
    wg, wu = x["wg"].double(), x["wu"].double()
    dx, dwg, dwu = torch.empty((m, c["dim"]), dtype=torch.float64, device="cuda"), torch.zeros_like(wg), torch.zeros_like(wu)
    step = max(1, (1 << 27) // c["hidden"])
    for a in range(0, m, step):
        v, dh = x["x"][a:a + step].double(), x["dh"][a:a + step].double()
        with torch.enable_grad():
            gate = x["gate"][a:a + step].double().requires_grad_()
            value = _act64(c["activation"], gate)
            dgate, = torch.autograd.grad(value, gate, dh * x["up"][a:a + step].double())
        dup = dh * value.detach()
        dx[a:a + step] = torch.einsum("mf,fd->md", dgate, wg) + torch.einsum("mf,fd->md", dup, wu)
        dwg += torch.einsum("mf,md->fd", dgate, v)
        dwu += torch.einsum("mf,md->fd", dup, v)
    return {"dx": dx, "dwg": dwg, "dwu": dwu}
