"""Plain forms of the 4-bit operands, written from the definition in sparsp.h, in 64 bits."""
import torch

BLOCK = {"mxfp4": 32, "nvfp4": 16}
LADDER = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def floor_log2(v):
    return torch.frexp(v)[1].double() - 1


def scale_codes(x, fmt, exponent):
    """[rows][blocks] codes of the scales of x [rows][cols]."""
    most = x.double().abs().unflatten(-1, (-1, BLOCK[fmt])).amax(-1)
    finite = most.isfinite()
    most = torch.where(finite, most, torch.ones_like(most))
    if fmt == "mxfp4":
        k = floor_log2(most / 6)
        k = torch.where(torch.exp2(k) * 6 < most, k + 1, k)
        code = torch.where(most == 0, torch.zeros_like(k), (k + 127).clamp(0, 254))
        return torch.where(finite, code, torch.full_like(code, 255)).to(torch.uint8)
    need = most / 6 * 2.0 ** -exponent
    e = floor_log2(need.clamp(min=2.0 ** -60)).clamp(min=-6)
    steps = (need / torch.exp2(e - 3)).round()  # 8 .. 16, less below 2^-6
    e, steps = torch.where(steps == 16, e + 1, e), torch.where(steps == 16, 8 * torch.ones_like(steps), steps)
    code = torch.where(steps < 8, steps, (e + 7) * 8 + steps - 8).clamp(max=126)
    return torch.where(finite, code, torch.full_like(code, 127)).to(torch.uint8)


def scale_values(codes, fmt, exponent):
    c = codes.double()
    if fmt == "mxfp4":
        return torch.where(c == 255, torch.full_like(c, float("nan")), torch.exp2(c - 127))
    e, m = (c / 8).floor(), c % 8
    v = torch.where(e == 0, m * 2.0 ** -9, (8 + m) * torch.exp2(e - 10))
    return torch.where(c == 127, torch.full_like(c, float("nan")), v * 2.0 ** exponent)


def quantize(x, fmt, exponent=0):
    """-> codes of the scales [rows][blocks], codes [rows][cols] 0 .. 15, what they stand for in 64 bits"""
    scales = scale_codes(x, fmt, exponent)
    s = scale_values(scales, fmt, exponent).unsqueeze(-1)
    v = x.double().unflatten(-1, (-1, BLOCK[fmt]))
    q = torch.where(s == 0, torch.zeros_like(v), v.abs() / s)
    code = torch.zeros_like(q, dtype=torch.int64)
    for i in range(7):
        middle = (LADDER[i] + LADDER[i + 1]) / 2
        code += (q > middle) if i % 2 == 0 else (q >= middle)
    ladder = torch.tensor(LADDER, dtype=torch.float64, device=x.device)
    values = ladder[code] * torch.where(v < 0, -1.0, 1.0) * s
    code = code + 8 * torch.signbit(v)
    return scales, code.flatten(-2), values.flatten(-2)


def unpack_codes(codes):
    """bytes [rows][cols / 2] -> [rows][cols]"""
    return torch.stack((codes & 15, codes >> 4), -1).flatten(-2)


def scale_places(rows, cols, fmt):
    """Where the scale of (row, block) lies, [rows][blocks], and how many bytes there are."""
    blocks = cols // BLOCK[fmt]
    groups = -(-blocks // 4)
    r, b = torch.arange(rows)[:, None], torch.arange(blocks)[None]
    at = (r // 128 * groups + b // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + b % 4
    return at, -(-rows // 128) * groups * 512
