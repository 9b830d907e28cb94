"""The norm of a list of gradients and their clipping against 64 bits.

A thread adds up to 32 squares in fp32 (each off by 2^-24 of itself and 31 additions of the sum so far), the rest is in
fp64: the sum is within 33 2^-24 of itself, the norm within half of that and a rounding to fp32.  A clipped value is its
gradient times a factor that is as far off as the norm, and a rounding of the factor, one of the product in fp32 and one to
its type."""
import math

import pytest
import torch

from layer_reference import F32, TINY, UNIT, close
from paper_2609_32197_b200 import binding

pytestmark = pytest.mark.gpu
BF, HF, FL = torch.bfloat16, torch.float16, torch.float32


def tensors(sizes, dtype, seed=0, scale=1.0, gap=0):
    """Views of one buffer, each `gap` elements behind the last: any alignment."""
    gen = torch.Generator().manual_seed(seed)
    buffer = (scale * torch.randn(sum(sizes) + gap * (len(sizes) + 1), generator=gen)).to(dtype).cuda()
    out, at = [], gap
    for n in sizes:
        out.append(buffer[at:at + n])
        at += n + gap
    return out


def norm_of(grads):
    return math.sqrt(math.fsum(float(g.double().square().sum()) for g in grads))


def clip(grads, limit, outs=None, ws=None, norm=True):
    ws = binding.make_grad_workspace() if ws is None else ws
    found = torch.full((1,), float("nan"), device="cuda") if norm else None
    lst = binding.make_grad_list(grads, outs)
    binding.sparsp_grad_squares(lst, ws)
    binding.sparsp_grad_clip(lst, limit, found, ws)
    return found


def check(got, grads, limit, norm, dtype):
    factor = min(1.0, limit / (norm + 1e-6))
    for g, w in zip(got, grads):
        want = w.double() * factor
        off = 19 * F32 * want.abs()
        close(g, want, off + UNIT[dtype] * (want.abs() + off) + TINY[dtype], "clipped")


SIZES = [[1], [7], [8], [9], [0, 5, 0], [8191], [8192], [8193], [4096, 4097, 1], [100003, 3, 64, 1, 70000], [1] * 64,
         [5, 17, 300] * 40, [33] * 1024, [33] * 1025, [11, 1000] * 1200, [3000017, 12]]


@pytest.mark.parametrize("dtype", [BF, HF, FL])
@pytest.mark.parametrize("gap", [0, 1, 8])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
def test_clip(sizes, gap, dtype):
    grads = tensors(sizes, dtype, len(sizes) + gap, 1.0, gap)
    norm, keep = norm_of(grads), [g.clone() for g in grads]
    for limit in (0.3 * norm, 3.0 * norm + 1.0, math.inf):
        outs = [torch.full_like(g, 7.0) for g in grads]
        got = clip(grads, limit, outs)
        assert abs(float(got) - norm) <= 18 * F32 * norm
        check(outs, grads, limit, norm, dtype)
        assert all(torch.equal(a, b) for a, b in zip(grads, keep))
        clip(grads, limit)  # in place: the same bits
        assert all(torch.equal(a, b) for a, b in zip(grads, outs))
        for g, k in zip(grads, keep):
            g.copy_(k)


def test_outputs_of_other_alignment():
    grads, outs = tensors([1001, 8200, 3], BF, 1, 1.0, 0), tensors([1001, 8200, 3], BF, 2, 1.0, 3)
    around = outs[0]._base.clone()
    norm = norm_of(grads)
    clip(grads, norm / 7, outs)
    check(outs, grads, norm / 7, norm, BF)
    at = 3
    for n in (1001, 8200, 3):
        around[at:at + n] = outs[0]._base[at:at + n]
        at += n + 3
    assert torch.equal(outs[0]._base, around)  # nothing beside them


@pytest.mark.parametrize("scale", [1e-30, 1e-20, 1e18, 1e30])
def test_squares_beyond_fp32(scale):
    grads = tensors([5000, 77], FL, 3, scale)
    norm = norm_of(grads)
    outs = [torch.empty_like(g) for g in grads]
    got = clip(grads, norm / 4 if norm > 1 else 1.0, outs)
    assert abs(float(got) - norm) <= 18 * F32 * norm
    check(outs, grads, norm / 4 if norm > 1 else 1.0, norm, FL)


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_a_norm_that_is_not_finite_changes_nothing(bad):
    grads = tensors([300, 9000], BF, 4)
    grads[1][8999] = bad
    keep = [g.clone() for g in grads]
    got = clip(grads, 1.0)
    assert not math.isfinite(float(got))
    for g, k in zip(grads, keep):
        assert torch.equal(g.view(torch.int16), k.view(torch.int16))
    outs = [torch.zeros_like(g) for g in grads]
    clip(grads, 1.0, outs)
    assert torch.equal(outs[0], keep[0]) and torch.equal(outs[1][:8999], keep[1][:8999])


def test_all_zero_and_no_gradients():
    grads = [torch.zeros(10000, device="cuda"), torch.zeros(3, device="cuda")]
    assert float(clip(grads, 1.0)) == 0.0 and not bool(grads[0].any())
    assert float(clip([], 1.0)) == 0.0


def test_several_types_share_one_norm():
    a, b = tensors([1000, 33], BF, 5), tensors([5000], FL, 6)
    ws, norm = binding.make_grad_workspace(), torch.empty(1, device="cuda")
    la, lb = binding.make_grad_list(a), binding.make_grad_list(b)
    want = norm_of(a + b)
    keep = [g.clone() for g in a + b]
    binding.sparsp_grad_squares(la, ws)
    binding.sparsp_grad_squares(lb, ws, accumulate=True)
    assert abs(float(binding.grad_square_sum(ws)) - want ** 2) <= 34 * F32 * want ** 2
    binding.sparsp_grad_clip(la, 2.0, norm, ws)
    binding.sparsp_grad_clip(lb, 2.0, None, ws)
    assert abs(float(norm) - want) <= 18 * F32 * want
    check(a, keep[:2], 2.0, want, BF)
    check(b, keep[2:], 2.0, want, FL)


def test_a_workspace_used_again_and_in_a_graph():
    """Lists of different lengths through one workspace, and a captured call replayed on new values."""
    ws = binding.make_grad_workspace()
    for n in (1, 1500, 3, 2000, 64):
        grads = tensors([50] * n, BF, n)
        norm = norm_of(grads)
        assert abs(float(clip(grads, math.inf, ws=ws)) - norm) <= 18 * F32 * norm
    grads = tensors([4000, 129], FL, 9)
    lst, norm = binding.make_grad_list(grads), torch.empty(1, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.sparsp_grad_squares(lst, ws)
        binding.sparsp_grad_clip(lst, 1.0, norm, ws)
    for seed in (10, 11):
        fresh = tensors([4000, 129], FL, seed)
        for g, f in zip(grads, fresh):
            g.copy_(f)
        graph.replay()
        want = norm_of(fresh)
        assert abs(float(norm) - want) <= 18 * F32 * want
        check(grads, fresh, 1.0, want, FL)


def test_same_bits():
    grads = tensors([1 << 20, 12345, 7], BF, 12)
    ws = binding.make_grad_workspace()
    lst = binding.make_grad_list(grads)
    sums = set()
    for _ in range(5):
        binding.sparsp_grad_squares(lst, ws)
        sums.add(float(binding.grad_square_sum(ws)))
    assert len(sums) == 1
