"""The work that the operators between a layer's products are judged by: 4-bit floating point operands with a scale for each
small block and their product, the gated residual step with its norms, and the clipping of a layer's gradients.

A case is a dict of plain values.  `op` says which call one pass makes:

  quantize   a matrix to 4-bit values with a scale for every 32 (mxfp4) or 16 (nvfp4) of a row; the values it then stands for
  product    C = A B^T + bias of two such operands
  step_fwd   r = x + gate * norm_y(y), n = norm_r(r) * weight + bias, with the row statistics that training keeps, or without
  step_bwd   its gradients: dx, dy and those of the gate and of every weight, summed over the rows that share it
  clip       the norm over a list of gradients, and the gradients times what brings it down to a limit

`own` chooses between the plain form (elementary torch operations in 32 bits, rounded once) and the library's calls.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}
BLOCK = {"mxfp4": 32, "nvfp4": 16}
EPS = 1e-5


def _quantize(name, rows, cols, *, fmt="mxfp4", dtype="bf16"):
    return {"name": name, "op": "quantize", "rows": rows, "cols": cols, "format": fmt, "dtype": dtype}


def _product(name, rows, cols, depth, *, fmt="mxfp4", dtype="bf16", bias=True):
    return {"name": name, "op": "product", "rows": rows, "cols": cols, "depth": depth, "format": fmt, "dtype": dtype, "bias": bias}


def _step(name, op, rows, dim, *, groups=1, norm_y="none", norm_r="layer", dtype="bf16", weights="fp32", stats=True):
    return {"name": name, "op": op, "rows": rows, "dim": dim, "groups": groups, "norm_y": norm_y, "norm_r": norm_r,
            "dtype": dtype, "weights": weights, "stats": stats}


def _clip(name, count, largest, *, values=0, spread=0, dtype="bf16", over=True):
    return {"name": name, "op": "clip", "count": count, "largest": largest, "values": values, "spread": spread, "dtype": dtype,
            "over": over}


def listed():
    return [
        # the hidden states of a long video layer before a projection
        _quantize("quantize-wan", 75600, 5120),
        # a feed-forward weight of such a layer, once for each optimiser step of training in 4 bits
        _quantize("quantize-weight", 13824, 5120, fmt="nvfp4"),
        # one sequence's condition to the six modulation vectors of a layer: every weight is read for one row
        _product("product-condition", 1, 6 * 5120, 5120, fmt="nvfp4"),
        # the text tokens of one prompt
        _product("product-text", 226, 7680, 1920, dtype="fp16"),
        # a long video layer's feed-forward projection: the largest case
        _product("product-wan", 75600, 13824, 5120, fmt="nvfp4"),
        # the smallest layer in use: latency
        _step("step-tiny", "step_fwd", 4096, 128, stats=False),
        # a long video layer between its halves, as training calls it
        _step("step-wan", "step_fwd", 75600, 5120),
        # its backward pass
        _step("step-wan-back", "step_bwd", 75600, 5120),
        # two sequences with weights of their own, the block's output normed too, in 32 bits
        _step("step-two-norms-back", "step_bwd", 2 * 7777, 1928, groups=2, norm_y="rms", norm_r="rms", dtype="fp32"),
        # the gradients of one long video layer's matrices and vectors
        _clip("clip-layer", 7, 13824 * 5120, values=4 * 5120 * 5120 + 3 * 13824 * 5120),
        # a model's many small tensors of odd sizes, under the limit
        _clip("clip-many", 300, 200003, spread=1, dtype="fp32", over=False),
    ]


def _log_int(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(("quantize", "product", "product", "step_fwd", "step_bwd", "clip"))
    dtype, fmt = rng.choice(("bf16", "bf16", "fp16", "fp32")), rng.choice(("mxfp4", "nvfp4"))
    if op == "quantize":
        cols = 32 * _log_int(rng, 1, 432)
        return _quantize("", _log_int(rng, 1, max(1, min(75600, 75600 * 5120 // cols))), cols, fmt=fmt, dtype=dtype)
    if op == "product":
        return _product("", _log_int(rng, 1, 75600), 8 * _log_int(rng, 1, 1728), 32 * _log_int(rng, 1, 160), fmt=fmt, dtype=dtype,
                        bias=rng.random() < 0.5)
    if op == "clip":
        return _clip("", _log_int(rng, 1, 500), _log_int(rng, 1, 1 << 20), spread=rng.randint(1, 1 << 20), dtype=dtype,
                     over=rng.random() < 0.7)
    dim, groups = 8 * _log_int(rng, 2, 1024), rng.choice((1, 1, 2, 5))
    per_group = _log_int(rng, 1, max(1, min(75600, 75600 * 5120 // dim // (2 if dtype == "fp32" else 1)) // groups))
    return _step("", op, groups * per_group, dim, groups=groups, norm_y=rng.choice(("none", "none", "layer", "rms")),
                 norm_r=rng.choice(("none", "layer", "layer", "rms")), dtype=dtype, weights=rng.choice((dtype, "fp32")),
                 stats=op == "step_bwd" or rng.random() < 0.6)


# ---- inputs ---------------------------------------------------------------------------------------------------------


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(gen, shape, dtype, scale=1.0):
    out = torch.empty(shape, dtype=dtype, device="cuda")
    return out.normal_(0.0, scale, generator=gen)


def _sizes(c):
    """Values of each tensor of a list of gradients, and where it begins in their common buffer."""
    if c["values"]:  # square matrices and three feed-forward ones: a layer
        rest = [c["largest"]] * 3
        sizes = rest + [(c["values"] - sum(rest)) // (c["count"] - 3)] * (c["count"] - 3)
    else:
        rng = random.Random(c["spread"])
        sizes = [c["largest"]] + [_log_int(rng, 1, c["largest"]) for _ in range(c["count"] - 1)]
    begins, at = [], 0
    for n in sizes:
        begins.append(at)
        at = (at + n + 63) // 64 * 64
    return sizes, begins, at


def _hidden_states(gen, rows, dim, dtype):
    """Channels of different sizes, a few of them far larger than the rest."""
    size = torch.empty(dim, device="cuda").normal_(0.0, 0.5, generator=gen).exp_()
    size[torch.randint(0, dim, (max(1, dim // 256),), generator=gen, device="cuda")] *= 8.0
    return _normal(gen, (rows, dim), dtype).mul_(size.to(dtype))


def _tensor_exponent(c, x):
    """The power of two that brings the largest block scale of nvfp4 into its 8 bits."""
    return math.ceil(math.log2(max(float(x.abs().max()), 2.0 ** -60) / (6 * 448))) if c["format"] == "nvfp4" else 0


def _inputs(c, seed):
    gen = _generator(seed)
    dt = DTYPES[c["dtype"]]
    if c["op"] == "quantize":
        x = {"x": _hidden_states(gen, c["rows"], c["cols"], dt)}
        x["exponent"] = _tensor_exponent(c, x["x"])
        return x
    if c["op"] == "product":
        x = {"a": _hidden_states(gen, c["rows"], c["depth"], torch.bfloat16),
             "b": _normal(gen, (c["cols"], c["depth"]), torch.bfloat16, c["depth"] ** -0.5)}
        x["exponent_a"], x["exponent_b"] = _tensor_exponent(c, x["a"]), _tensor_exponent(c, x["b"])
        if c["bias"]:
            x["bias"] = _normal(gen, (c["cols"],), dt)
        return x
    if c["op"] == "clip":
        sizes, begins, total = _sizes(c)
        x = {"g": _normal(gen, (total,), dt, 1e-3)}
        for n, at in zip(sizes, begins):
            x["g"][at + n:(at + n + 63) // 64 * 64] = 0
        x["limit"] = 1e-3 * math.sqrt(sum(sizes)) * (0.37 if c["over"] else 2.0)
        return x
    rows, dim, groups, wt = c["rows"], c["dim"], c["groups"], DTYPES[c["weights"]]
    x = {"y": _normal(gen, (rows, dim), dt, 0.7), "gate": _normal(gen, (groups, dim), wt, 0.5)}
    if c["norm_y"] != "none":
        x["wy"], x["by"] = _normal(gen, (dim,), torch.float32, 0.2).add_(1.0).to(wt), _normal(gen, (dim,), wt, 0.2)
    if c["norm_r"] != "none":
        x["wr"] = _normal(gen, (groups, dim), torch.float32, 0.2).add_(1.0).to(wt)
        x["br"] = _normal(gen, (groups, dim), wt, 0.2)
    if c["op"] == "step_fwd":
        x["x"] = _hidden_states(gen, rows, dim, dt).add_(0.5)
        return x
    x["r"] = _hidden_states(gen, rows, dim, dt).add_(0.5)
    x["dr"] = _normal(gen, (rows, dim), dt)
    x["stats_y"], x["stats_r"] = (_statistics(c[k], x[v]) for k, v in (("norm_y", "y"), ("norm_r", "r")))
    if c["norm_r"] != "none":
        x["dn"] = _normal(gen, (rows, dim), dt)
    return x


def _statistics(kind, v):
    """[rows][2] (mean, 1 / deviation) that the forward pass kept of v."""
    if kind == "none":
        return None
    out = torch.empty((v.shape[0], 2), device="cuda")
    step = max(1, (1 << 27) // v.shape[1])
    for r in range(0, v.shape[0], step):
        part = v[r:r + step].double()
        mean = part.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(part[:, :1])
        out[r:r + step] = torch.cat((mean, ((part - mean).square().mean(1, keepdim=True) + EPS).rsqrt()), 1)
    return out


def prepare(case, seed):
    c = dict(case)
    x = _inputs(c, seed)
    if own:
        _plan(c, x)
    elif c["op"] == "product":  # both operands are in 4 bits before the call: here as the values they stand for
        x["a"], x["b"] = _plain_values(c, x["a"], x["exponent_a"]), _plain_values(c, x["b"], x["exponent_b"])
    return c, x


def _plan(c, x):
    """What a program of the library keeps beside its data: descriptions, operands, buffers for results, a workspace."""
    from paper_2609_32197_b200 import binding

    dt = DTYPES[c["dtype"]]
    if c["op"] == "quantize":
        x["fp4"] = binding.make_fp4(c["rows"], c["cols"], c["format"], x["exponent"], dt)
        x["operand"] = binding.make_fp4_operand(x["fp4"])
        x["out"] = {"values": torch.empty_like(x["x"])}
    elif c["op"] == "product":
        for k, rows in (("a", c["rows"]), ("b", c["cols"])):
            fp4 = binding.make_fp4(rows, c["depth"], c["format"], x["exponent_" + k], torch.bfloat16)
            matrix = x[k]
            x[k] = binding.make_fp4_operand(fp4)
            binding.sparsp_fp4_quantize(fp4, matrix, *x[k], None)
        x["product"] = binding.make_fp4_product(c["rows"], c["cols"], c["depth"], c["format"], x["exponent_a"] + x["exponent_b"], dt)
        x["workspace"] = binding.make_fp4_product_workspace(x["product"])
        x["out"] = {"c": torch.empty((c["rows"], c["cols"]), dtype=dt, device="cuda")}
    elif c["op"] == "clip":
        sizes, begins, _ = _sizes(c)
        x["out"] = {"g": torch.zeros_like(x["g"]), "norm": torch.empty(1, device="cuda")}
        x["list"] = binding.make_grad_list([x["g"][a:a + n] for n, a in zip(sizes, begins)],
                                           [x["out"]["g"][a:a + n] for n, a in zip(sizes, begins)])
        x["workspace"] = binding.make_grad_workspace()
    else:
        x["step"] = binding.make_gated_norm(c["rows"], c["dim"], rows_per_group=c["rows"] // c["groups"], norm_y=c["norm_y"],
                                            norm_r=c["norm_r"], eps=EPS, dtype=dt, weight_dtype=DTYPES[c["weights"]])
        if c["op"] == "step_fwd":
            x["out"] = {"r": torch.empty_like(x["x"])}
            if c["norm_r"] != "none":
                x["out"]["n"] = torch.empty_like(x["x"])
            if c["stats"]:
                for k in ("y", "r"):
                    if c["norm_" + k] != "none":
                        x["out"]["stats_" + k] = torch.empty((c["rows"], 2), device="cuda")
        else:
            x["out"] = {"d" + k: torch.empty_like(x[k]) for k in ("y", "gate", "wy", "by", "wr", "br") if k in x}
            x["out"]["dx"] = torch.empty_like(x["r"])
            x["workspace"] = binding.make_gated_norm_workspace(x["step"])


# ---- one pass -------------------------------------------------------------------------------------------------------


def run(state):
    c, x = state
    if own:
        return _run_own(c, x)
    return {"quantize": _plain_quantize, "product": _plain_product, "step_fwd": _plain_step_fwd, "step_bwd": _plain_step_bwd,
            "clip": _plain_clip}[c["op"]](c, x)


def _run_own(c, x):
    from paper_2609_32197_b200 import binding

    o = x["out"]
    if c["op"] == "quantize":
        binding.sparsp_fp4_quantize(x["fp4"], x["x"], *x["operand"], o["values"])
    elif c["op"] == "product":
        binding.sparsp_fp4_product(x["product"], *x["a"], *x["b"], x.get("bias"), o["c"], x["workspace"])
    elif c["op"] == "step_fwd":
        binding.sparsp_gated_norm_fwd(x["step"], x["x"], x["y"], x["gate"], x.get("wy"), x.get("by"), x.get("wr"), x.get("br"),
                                      o["r"], o.get("n"), o.get("stats_y"), o.get("stats_r"))
    elif c["op"] == "step_bwd":
        r = x["r"] if c["norm_r"] != "none" else None
        binding.sparsp_gated_norm_bwd(x["step"], x.get("dn"), x["dr"], r, x["y"], x["gate"], x.get("wy"), x.get("by"),
                                      x.get("wr"), x["stats_y"], x["stats_r"], o["dx"], o["dy"], o["dgate"], o.get("dwy"),
                                      o.get("dby"), o.get("dwr"), o.get("dbr"), x["workspace"])
    else:
        binding.sparsp_grad_squares(x["list"], x["workspace"])
        binding.sparsp_grad_clip(x["list"], x["limit"], o["norm"], x["workspace"])
    return o


def _plain_values(c, x, exponent):
    """The values that a matrix stands for after rounding to 4 bits, in 32 bits."""
    v = x.float().unflatten(-1, (-1, BLOCK[c["format"]]))
    most = v.abs().amax(-1, keepdim=True)
    if c["format"] == "mxfp4":  # the least power of two with which the block's largest is at most 6
        m, e = torch.frexp(most)
        scale = torch.exp2((e - 3 + (m > 0.75)).double().clamp(-127, 127))
    else:
        scale = (most * 2.0 ** -exponent / 6).clamp(max=448).to(torch.float8_e4m3fn).double() * 2.0 ** exponent
    scale = torch.where(most == 0, torch.zeros_like(scale), scale).float()
    q = torch.where(scale == 0, torch.zeros_like(v), v / scale)
    step = 0.5 + 0.5 * (q.abs() >= 2) + (q.abs() >= 4)  # between neighbours of 0, 0.5, 1, 1.5, 2, 3, 4, 6
    return ((q / step).round() * step).clamp(-6, 6).mul(scale).flatten(-2)


def _plain_quantize(c, x):
    return {"values": _plain_values(c, x["x"], x["exponent"]).to(x["x"].dtype)}


def _plain_product(c, x):
    y = x["a"] @ x["b"].T
    return {"c": (y + x["bias"].float() if c["bias"] else y).to(DTYPES[c["dtype"]])}


def _rows(c, v):
    """[groups][rows of a group][dim] in 32 bits."""
    return v.float().view(c["groups"], -1, v.shape[-1])


def _per_row(w):
    """A weight of each group against the rows of its group, in 32 bits."""
    return w.float()[:, None, :]


def _normed(kind, v):
    """v normed along its last dimension, and its [rows][2] statistics."""
    mean = v.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(v[..., :1])
    v = v - mean
    rstd = (v.square().mean(-1, keepdim=True) + EPS).rsqrt()
    return v * rstd, torch.cat((mean, rstd), -1).view(-1, 2)


def _plain_step_fwd(c, x):
    out, u = {}, _rows(c, x["y"])
    if c["norm_y"] != "none":
        u, stats = _normed(c["norm_y"], u)
        u = u * x["wy"].float() + x["by"].float()
        if c["stats"]:
            out["stats_y"] = stats
    r = _rows(c, x["x"]) + _per_row(x["gate"]) * u
    out["r"] = r.to(x["x"].dtype).view_as(x["x"])
    if c["norm_r"] != "none":
        n, stats = _normed(c["norm_r"], r)
        out["n"] = (n * _per_row(x["wr"]) + _per_row(x["br"])).to(x["x"].dtype).view_as(x["x"])
        if c["stats"]:
            out["stats_r"] = stats
    return out


def _normed_again(c, v, stats):
    s = stats.view(c["groups"], -1, 2)
    return (_rows(c, v) - s[..., :1]) * s[..., 1:]


def _through_norm(c, kind, a, vh, stats):
    """The gradient of what a norm took, for a at its result before the weights."""
    along = vh * (a * vh).mean(-1, keepdim=True)
    return (a - along - (a.mean(-1, keepdim=True) if kind == "layer" else 0.0)) * stats.view(c["groups"], -1, 2)[..., 1:]


def _plain_step_bwd(c, x):
    out, t, shape, dt, wt = {}, _rows(c, x["dr"]), x["r"].shape, x["r"].dtype, x["gate"].dtype
    if c["norm_r"] != "none":
        dn, rh = _rows(c, x["dn"]), _normed_again(c, x["r"], x["stats_r"])
        t = t + _through_norm(c, c["norm_r"], dn * _per_row(x["wr"]), rh, x["stats_r"])
        out["dwr"], out["dbr"] = (dn * rh).sum(1).to(wt), dn.sum(1).to(wt)
        del dn, rh
    out["dx"] = t.to(dt).view(shape)
    du = t * _per_row(x["gate"])
    if c["norm_y"] == "none":
        out["dgate"] = (t * _rows(c, x["y"])).sum(1).to(wt)
    else:
        yh = _normed_again(c, x["y"], x["stats_y"])
        out["dgate"] = (t * (yh * x["wy"].float() + x["by"].float())).sum(1).to(wt)
        out["dwy"], out["dby"] = (du * yh).sum((0, 1)).to(wt), du.sum((0, 1)).to(wt)
        du = _through_norm(c, c["norm_y"], du * x["wy"].float(), yh, x["stats_y"])
    out["dy"] = du.to(dt).view(shape)
    return out


def _plain_clip(c, x):
    norm = x["g"].float().square().sum(dtype=torch.float64).sqrt()
    factor = (x["limit"] / (norm + 1e-6)).clamp(max=1.0).float()
    return {"g": (x["g"].float() * factor).to(x["g"].dtype), "norm": norm.float().view(1)}


# ---- what a pass cannot do without ----------------------------------------------------------------------------------


def _fp4_bytes(c, rows, cols):
    return rows * cols // 2 + rows * cols // BLOCK[c["format"]]


def work(case):
    c = case
    e = BYTES[c["dtype"]]
    if c["op"] == "quantize":
        return {"bytes": 2 * e * c["rows"] * c["cols"] + _fp4_bytes(c, c["rows"], c["cols"]), "flops": 4 * c["rows"] * c["cols"]}
    if c["op"] == "product":
        m, n, k = c["rows"], c["cols"], c["depth"]
        return {"bytes": _fp4_bytes(c, m, k) + _fp4_bytes(c, n, k) + e * (m * n + (n if c["bias"] else 0)), "flops": 2 * m * n * k}
    if c["op"] == "clip":
        values = sum(_sizes(c)[0])
        return {"bytes": 2 * e * values, "flops": 3 * values}
    size, wsize = c["rows"] * c["dim"], c["dim"] * BYTES[c["weights"]]
    y, r = c["norm_y"] != "none", c["norm_r"] != "none"
    weights = wsize * (c["groups"] * (3 if r else 1) + (2 if y else 0))
    kept = 8 * c["rows"] * (y + r) if c["stats"] else 0
    if c["op"] == "step_fwd":
        return {"bytes": size * e * (4 if r else 3) + weights + kept, "flops": size * (2 + 8 * (y + r))}
    return {"bytes": size * e * (6 if r else 4) + 2 * weights + kept, "flops": size * (4 + 13 * (y + r))}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------


def exact(case, seed):
    c = dict(case)
    x = _inputs(c, seed)
    return {"quantize": _exact_quantize, "product": _exact_product, "step_fwd": _exact_step_fwd, "step_bwd": _exact_step_bwd,
            "clip": _exact_clip}[c["op"]](c, x)


def _floor_log2(v):
    return torch.frexp(v)[1].double() - 1


def _exact_values(c, x, exponent):
    """Part by part: the nearest of the eight magnitudes, a tie to the one whose code is even."""
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    ladder = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=x.device)
    step = max(1, (1 << 25) // x.shape[1])
    for a in range(0, x.shape[0], step):
        v = x[a:a + step].double().unflatten(-1, (-1, BLOCK[c["format"]]))
        need = v.abs().amax(-1, keepdim=True) / 6
        if c["format"] == "mxfp4":
            k = _floor_log2(need)
            scale = torch.exp2(torch.where(torch.exp2(k) < need, k + 1, k).clamp(min=-127))
        else:
            need = need * 2.0 ** -exponent
            unit = torch.exp2(_floor_log2(need).clamp(min=-6) - 3)
            scale = (need / unit).round().mul(unit).clamp(max=448.0) * 2.0 ** exponent
        scale = torch.where(need == 0, torch.zeros_like(scale), scale)
        q = torch.where(scale == 0, torch.zeros_like(v), v.abs() / scale)
        code = torch.zeros_like(q, dtype=torch.int64)
        for i in range(7):
            middle = (ladder[i] + ladder[i + 1]) / 2
            code += (q > middle) if i % 2 == 0 else (q >= middle)
        out[a:a + step] = (ladder[code] * torch.sign(v) * scale).flatten(-2)
    return out


def _exact_quantize(c, x):
    return {"values": _exact_values(c, x["x"], x["exponent"])}


def _exact_product(c, x):
    a, b = _exact_values(c, x["a"], x["exponent_a"]), _exact_values(c, x["b"], x["exponent_b"])
    y = torch.einsum("mk,nk->mn", a, b)
    return {"c": y.add_(x["bias"].double()) if c["bias"] else y}


def _chunks(c):
    """Rows [a, b) of one group at a time, few enough to be held in 64 bits several times over."""
    per, step = c["rows"] // c["groups"], max(1, (1 << 27) // c["dim"])
    for g in range(c["groups"]):
        for a in range(g * per, (g + 1) * per, step):
            yield g, a, min(a + step, (g + 1) * per)


def _exact_norm(kind, v):
    if kind == "layer":
        var, mean = torch.var_mean(v, 1, unbiased=False, keepdim=True)
        return (v - mean) / torch.sqrt(var + EPS), torch.cat((mean, 1 / torch.sqrt(var + EPS)), 1)
    size = torch.sqrt(torch.einsum("rd,rd->r", v, v)[:, None] / v.shape[1] + EPS)
    return v / size, torch.cat((torch.zeros_like(size), 1 / size), 1)


def _exact_step_fwd(c, x):
    found = {}
    for g, a, b in _chunks(c):
        u, part = x["y"][a:b].double(), {}
        if c["norm_y"] != "none":
            u, part["stats_y"] = _exact_norm(c["norm_y"], u)
            u = torch.addcmul(x["by"].double(), u, x["wy"].double())
        part["r"] = torch.addcmul(x["x"][a:b].double(), u, x["gate"][g].double())
        if c["norm_r"] != "none":
            n, part["stats_r"] = _exact_norm(c["norm_r"], part["r"])
            part["n"] = torch.addcmul(x["br"][g].double(), n, x["wr"][g].double())
        for k, v in part.items():
            if c["stats"] or not k.startswith("stats"):
                found.setdefault(k, []).append(v)
    return {k: torch.cat(v) for k, v in found.items()}


def _exact_back(kind, a, v, stats):
    """(v normed by its kept statistics, gradient of v), row by row: the matrix (I - P) of each norm applied to a."""
    mean, rstd = stats[:, :1].double(), stats[:, 1:].double()
    vh = (v - mean) * rstd
    back = a - torch.einsum("rd,rd->r", a, vh)[:, None] / v.shape[1] * vh
    if kind == "layer":
        back = back - a.sum(1, keepdim=True) / v.shape[1]
    return vh, back * rstd


def _exact_step_bwd(c, x):
    rows, dim = x["r"].shape
    out = {k: torch.empty((rows, dim), dtype=torch.float64, device="cuda") for k in ("dx", "dy")}
    for k in ("gate", "wy", "by", "wr", "br"):
        if k in x:
            out["d" + k] = torch.zeros(x[k].shape, dtype=torch.float64, device="cuda")
    for g, a, b in _chunks(c):
        t, y, gate = x["dr"][a:b].double(), x["y"][a:b].double(), x["gate"][g].double()
        if c["norm_r"] != "none":
            dn = x["dn"][a:b].double()
            rh, back = _exact_back(c["norm_r"], dn * x["wr"][g].double(), x["r"][a:b].double(), x["stats_r"][a:b])
            t = t + back
            out["dwr"][g] += torch.einsum("rd,rd->d", dn, rh)
            out["dbr"][g] += dn.sum(0)
        out["dx"][a:b] = t
        if c["norm_y"] == "none":
            out["dy"][a:b] = t * gate
            out["dgate"][g] += torch.einsum("rd,rd->d", t, y)
        else:
            yh, out["dy"][a:b] = _exact_back(c["norm_y"], t * gate * x["wy"].double(), y, x["stats_y"][a:b])
            along, alone = torch.einsum("rd,rd->d", t, yh), t.sum(0)
            out["dgate"][g] += along * x["wy"].double() + alone * x["by"].double()
            out["dwy"] += along * gate
            out["dby"] += alone * gate
    return out


def _exact_clip(c, x):
    sizes, begins, _ = _sizes(c)
    norm = math.sqrt(math.fsum(float(torch.linalg.vector_norm(x["g"][a:a + n].double())) ** 2 for n, a in zip(sizes, begins)))
    return {"g": x["g"].double() * min(1.0, x["limit"] / (norm + 1e-6)),
            "norm": torch.tensor([norm], dtype=torch.float64, device="cuda")}
