"""Rotary positions against the plain 64-bit form.

Bound of an element: the rounding of the stored value, and in fp32 the rounding of c and s, of two products and of a sum,
each at most 2^-24 of amplitude * (|a| + |b|)."""
import pytest
import torch

from layer_reference import F32, TINY, UNIT, close, rotate
from paper_2609_32197_b200 import binding

pytestmark = pytest.mark.gpu


def make_case(B, H, grid, n_text, d, layout, dtype, seed=0):
    gen = torch.Generator().manual_seed(seed)
    N = grid[0] * grid[1] * grid[2] + n_text
    dims = (B, H, N, d) if layout == "HND" else (B, N, H, d)
    q, k = (torch.randn(dims, generator=gen).to(dtype).cuda() for _ in range(2))
    return binding.make_shape(H, d, grid, n_text, 64, batch=B, layout=layout), q, k


def as_hnd(x, layout):
    return (x if layout == "HND" else x.transpose(1, 2)).double()


def expected(x, layout, pairs, freq, amplitude, pos, rot_begin, half, inverse):
    """pos [B][N][3] int, rotated where the first is >= 0"""
    angle = torch.cat([pos[..., a:a + 1].double() * f.cuda() for a, f in enumerate(freq)], -1)
    return rotate(as_hnd(x, layout), amplitude * angle.cos(), amplitude * angle.sin(), pos[..., 0] >= 0, rot_begin, half,
                  inverse)


def grid_positions(grid, n_text, origin, B):
    t, h, w = torch.meshgrid(*(torch.arange(g) + o for g, o in zip(grid, origin)), indexing="ij")
    pos = torch.stack((t.reshape(-1), h.reshape(-1), w.reshape(-1)), 1)
    pos = torch.cat((pos, torch.full((n_text, 3), -1)))
    return pos.to(torch.int32).cuda()[None].expand(B, -1, -1).contiguous()


def bound_of(x, layout, want, dtype, amplitude):
    scale = as_hnd(x, layout).abs().amax(-1, keepdim=True) * 2 * amplitude
    return UNIT[dtype] * want.abs() + TINY[dtype] + 5 * F32 * scale


def frequencies(pairs, **kw):
    out, amplitude = [], 1.0
    for n in pairs:
        f, amplitude = binding.sparsp_rotary_frequencies(n, **kw)
        out.append(f)
    return out, amplitude


CASES = [
    # B, H, grid, text, d, pairs, rot_begin, layout, pairing, dtype
    (1, 2, (4, 5, 7), 0, 64, (16, 8, 8), 0, "HND", "interleaved", torch.bfloat16),
    (2, 3, (3, 4, 5), 11, 128, (22, 21, 21), 0, "NHD", "interleaved", torch.bfloat16),
    (1, 5, (3, 4, 5), 1, 64, (8, 8, 8), 0, "NHD", "half", torch.float16),
    (2, 1, (2, 3, 3), 3, 64, (8, 8, 8), 16, "HND", "half", torch.float32),
    (1, 7, (1, 1, 1), 0, 128, (32, 0, 0), 64, "NHD", "half", torch.bfloat16),
    (3, 9, (17, 1, 1), 0, 80, (20, 0, 0), 40, "HND", "interleaved", torch.bfloat16),
    (1, 4, (2, 3, 5), 2, 128, (5, 7, 9), 3, "HND", "half", torch.bfloat16),  # nothing on 16 bytes
    (1, 4, (2, 3, 5), 2, 128, (5, 7, 9), 3, "NHD", "interleaved", torch.float32),
    (1, 2, (2, 3, 5), 0, 256, (128, 0, 0), 0, "HND", "interleaved", torch.float16),
    (1, 2, (2, 3, 5), 0, 8, (0, 1, 0), 1, "HND", "half", torch.float32),
    (1, 1, (1, 37, 41), 5, 64, (0, 16, 16), 0, "NHD", "half", torch.bfloat16),
    (1, 41, (1, 9, 1), 0, 64, (1, 1, 0), 60, "NHD", "interleaved", torch.bfloat16),
]


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"B{c[0]}H{c[1]}d{c[4]}-{c[7]}-{c[8]}-{str(c[9])[6:]}")
def test_rotation_on_the_grid(case, inverse):
    B, H, grid, n_text, d, pairs, begin, layout, pairing, dtype = case
    shape, q, k = make_case(B, H, grid, n_text, d, layout, dtype)
    freq, amplitude = frequencies(pairs)
    rotary = binding.make_rotary(pairs, tuple(g + 9 for g in grid), pairing, begin, dtype)
    table = binding.make_rotary_table(rotary, torch.cat(freq), amplitude)
    origin = (4, 0, 9)
    qo, ko = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    binding.sparsp_rotary_apply(shape, rotary, table, None, origin, q, k, qo, ko, inverse, None)
    pos = grid_positions(grid, n_text, origin, B)
    for x, y in ((q, qo), (k, ko)):
        want = expected(x, layout, pairs, freq, amplitude, pos, begin, pairing == "half", inverse)
        close(as_hnd(y, layout), want, bound_of(x, layout, want, dtype, amplitude), "rotated")
    # in place, Q alone: the same bits
    alone = q.clone()
    binding.sparsp_rotary_apply(shape, rotary, table, None, origin, alone, None, alone, None, inverse, None)
    assert torch.equal(alone, qo)


@pytest.mark.parametrize("pairing", ["interleaved", "half"])
def test_positions_of_permuted_tokens(pairing):
    """Tokens in another order, with their positions, give the same rows in that order."""
    grid, n_text, pairs = (3, 8, 8), 7, (8, 12, 12)
    shape, q, k = make_case(1, 3, grid, n_text, 64, "HND", torch.bfloat16)
    freq, amplitude = frequencies(pairs)
    rotary = binding.make_rotary(pairs, grid, pairing)
    table = binding.make_rotary_table(rotary, torch.cat(freq), amplitude)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    binding.sparsp_rotary_apply(shape, rotary, table, None, (0, 0, 0), q, k, qo, ko, False, None)
    order = torch.randperm(q.shape[2], generator=torch.Generator().manual_seed(3)).cuda()
    pos = grid_positions(grid, n_text, (0, 0, 0), 1)[0][order].contiguous()
    qp, kp = q[:, :, order].contiguous(), k[:, :, order].contiguous()
    ws = binding.make_status_workspace()
    binding.sparsp_rotary_apply(shape, rotary, table, pos, (0, 0, 0), qp, kp, qp, kp, False, ws)
    assert torch.equal(qp, qo[:, :, order]) and torch.equal(kp, ko[:, :, order])
    assert binding.sparsp_status(ws) == binding.SPARSP_OK


@pytest.mark.parametrize("scaling,factor", [("none", 1.0), ("linear", 4.0), ("ntk", 8.0), ("yarn", 4.0)])
def test_long_contexts(scaling, factor):
    """One token of each of several requests, up to the end of a table of a million positions."""
    length, pairs, B, H, d = 1 << 20, (32, 0, 0), 5, 3, 64
    shape, q, _ = make_case(B, H, (1, 1, 1), 0, d, "NHD", torch.float32)
    freq, amplitude = frequencies(pairs, theta=500000.0, scaling=scaling, factor=factor, original_length=8192.0)
    rotary = binding.make_rotary(pairs, (length, 0, 0), "half", 0, torch.float32)
    table = binding.make_rotary_table(rotary, torch.cat(freq), amplitude)
    pos = torch.tensor([[[0, 5, 5]], [[1, 0, 0]], [[8191, 0, -4]], [[length - 1, 0, 0]], [[-1, 0, 0]]], dtype=torch.int32,
                       device="cuda")
    out, ws = torch.empty_like(q), binding.make_status_workspace()
    binding.sparsp_rotary_apply(shape, rotary, table, pos, (0, 0, 0), q, None, out, None, False, ws)
    want = expected(q, "NHD", pairs, freq, amplitude, pos, 0, True, False)
    close(as_hnd(out, "NHD"), want, bound_of(q, "NHD", want, torch.float32, amplitude), scaling)
    assert binding.sparsp_status(ws) == binding.SPARSP_OK
    assert torch.equal(out[4], q[4])


def test_a_position_outside_the_table_is_reported():
    shape, q, _ = make_case(1, 2, (4, 1, 1), 0, 64, "HND", torch.bfloat16)
    rotary = binding.make_rotary((8, 8, 0), (4, 3, 0))
    freq, _ = frequencies((8, 8))
    table = binding.make_rotary_table(rotary, torch.cat(freq))
    for bad in ([4, 0, 0], [0, 3, 0], [0, -1, 0], [2 ** 31 - 1, 0, 0]):
        pos = torch.tensor([[0, 0, 0], [3, 2, 99], bad, [-7, 99, 99]], dtype=torch.int32, device="cuda")
        out, ws = torch.empty_like(q), binding.make_status_workspace()
        binding.sparsp_rotary_apply(shape, rotary, table, pos, (0, 0, 0), q, None, out, None, False, ws)
        assert binding.sparsp_status(ws) == binding.SPARSP_ERR_INVALID_ARG
        assert torch.equal(out[:, :, 2:], q[:, :, 2:])  # it keeps its values, as does the one without a position
        assert torch.equal(out[:, :, :1], q[:, :, :1])  # position 0: the rotation by no angle
        assert not torch.equal(out[:, :, 1], q[:, :, 1])
        assert binding.sparsp_status(ws) == binding.SPARSP_OK


def test_padded_strides_and_untouched_gaps():
    B, H, grid, d = 2, 3, (2, 3, 5), 64
    N = 30
    big = torch.randn(B, H + 1, N + 2, d + 24, generator=torch.Generator().manual_seed(5)).to(torch.bfloat16).cuda()
    shape = binding.sparsp_shape(B, H, d, *grid, 0, 64, big.stride(0), big.stride(1), big.stride(2))
    pairs = (8, 8, 8)
    freq, amplitude = frequencies(pairs)
    rotary = binding.make_rotary(pairs, grid)
    table = binding.make_rotary_table(rotary, torch.cat(freq))
    out = big.clone()
    binding.sparsp_rotary_apply(shape, rotary, table, None, (0, 0, 0), big, None, out, None, False, None)
    x = big[:, :H, :N, :d]
    want = expected(x, "HND", pairs, freq, amplitude, grid_positions(grid, 0, (0, 0, 0), B), 0, False, False)
    close(out[:, :H, :N, :d], want, bound_of(x, "HND", want, torch.bfloat16, 1.0), "strided")
    same = torch.ones_like(big, dtype=torch.bool)
    same[:, :H, :N, :48] = False
    assert torch.equal(out[same], big[same])


def test_special_values_stay_in_their_pairs():
    shape, q, _ = make_case(1, 1, (3, 1, 1), 1, 64, "HND", torch.float32)
    q[0, 0, 1, 0] = float("nan")
    q[0, 0, 2, 3] = float("inf")
    q[0, 0, 3, 5] = float("inf")  # the text token: copied
    rotary = binding.make_rotary((32, 0, 0), (3, 0, 0), dtype=torch.float32)
    freq, _ = frequencies((32,))
    out = torch.empty_like(q)
    binding.sparsp_rotary_apply(shape, rotary, binding.make_rotary_table(rotary, freq[0]), None, (0, 0, 0), q, None, out,
                                None, False, None)
    bad = ~torch.isfinite(out[0, 0])
    assert bad.nonzero().tolist() == [[1, 0], [1, 1], [2, 2], [2, 3], [3, 5]]


@pytest.mark.parametrize("pairing", ["interleaved", "half"])
def test_the_inverse_is_the_gradient(pairing):
    """<R x, g> = <x, R' g> for the amplitude too, and differences of <R x, g> along any direction give <R' g, v>."""
    grid, pairs, d = (5, 6, 7), (8, 12, 12), 64
    shape, x, g = make_case(1, 2, grid, 3, d, "HND", torch.float32, seed=2)
    freq, amplitude = frequencies(pairs, scaling="yarn", factor=4.0, original_length=64.0)
    rotary = binding.make_rotary(pairs, grid, pairing, 0, torch.float32)
    table = binding.make_rotary_table(rotary, torch.cat(freq), amplitude)
    y, back = torch.empty_like(x), torch.empty_like(g)
    binding.sparsp_rotary_apply(shape, rotary, table, None, (0, 0, 0), x, None, y, None, False, None)
    binding.sparsp_rotary_apply(shape, rotary, table, None, (0, 0, 0), g, None, back, None, True, None)
    size = float((x.double().abs() * g.double().abs()).sum())
    assert abs(float((y.double() * g.double()).sum() - (x.double() * back.double()).sum())) <= 20 * F32 * size
    v = torch.randn(x.shape, generator=torch.Generator().manual_seed(9)).cuda()
    # the loss is linear in x, so a step of one is as good as a small one
    up, down = torch.empty_like(x), torch.empty_like(x)
    binding.sparsp_rotary_apply(shape, rotary, table, None, (0, 0, 0), x + v, None, up, None, False, None)
    binding.sparsp_rotary_apply(shape, rotary, table, None, (0, 0, 0), x - v, None, down, None, False, None)
    slope = float(((up.double() - down.double()) * g.double()).sum()) / 2
    size = float(((x.double().abs() + v.double().abs()) * g.double().abs()).sum())
    assert abs(slope - float((back.double() * v.double()).sum())) <= 40 * F32 * size
