"""The memory of a list's table stays its own until the calls on every stream are done, although the list is dropped before."""
import gc

import pytest
import torch

from paper_2609_32197_b200 import binding
from test_step_host import grads, table_of


class Table:
    def __init__(self):
        self.streams = []

    def data_ptr(self):
        return 1 << 16

    def record_stream(self, stream):
        self.streams.append(stream)


def test_a_call_on_another_stream_is_told_to_the_table(monkeypatch):
    lst = grads((4096, 8))
    binding.sparsp_grad_table(lst, table_of(lst))
    lst.table, lst.stream, calls = Table(), 7, []

    class Library:
        def sparsp_grad_squares(self, *args):
            calls.append(args[1:])
            return 0

        sparsp_grad_clip = sparsp_grad_squares

    monkeypatch.setattr(binding, "lib", lambda: Library())
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: "another")
    for stream, told in ((7, 0), (9, 2)):
        monkeypatch.setattr(binding, "_stream_handle", lambda: stream)
        binding.sparsp_grad_squares(lst, None)
        binding.sparsp_grad_clip(lst, 1.0, None, None)
        assert lst.table.streams == ["another"] * told
    assert calls[2:] == [(1 << 16, 0, None, 9), (1 << 16, 1.0, None, None, 9)]
    assert grads((4096, 8)).stream is None


@pytest.mark.gpu
def test_a_list_dropped_while_another_stream_runs_its_calls():
    g = torch.ones(5000, device="cuda")
    ws, norm, side = binding.make_grad_workspace(), torch.zeros(1, device="cuda"), torch.cuda.Stream()
    lst = binding.make_grad_list([g])
    binding.sparsp_grad_squares(lst, ws)  # (the first calls load the library and its kernels, which takes longer than the sleep)
    binding.sparsp_grad_clip(lst, 100.0, norm, ws)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)  # 0.1 s of clocks in front of the calls
        binding.sparsp_grad_squares(lst, ws)
        binding.sparsp_grad_clip(lst, 1.0, norm, ws)
    at, size = lst.table.data_ptr(), lst.table.numel()
    del lst
    gc.collect()
    others = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(8)]
    assert not side.query()
    assert all(o.data_ptr() + size <= at or at + size <= o.data_ptr() for o in others)
    side.synchronize()
    assert abs(float(norm) - 5000 ** 0.5) <= 1e-6 * 5000 ** 0.5


@pytest.mark.gpu
def test_a_list_made_again_on_new_addresses():
    """Gradients that are somewhere else after every step, as autograd gives them: a list for each step."""
    ws, norm = binding.make_grad_workspace(), torch.empty(1, device="cuda")
    weight = torch.randn(300, 70, generator=torch.Generator().manual_seed(1)).cuda().requires_grad_()
    held = []
    for step in range(5):
        weight.grad = None
        (weight * (step + 1.0)).square().sum().backward()
        want, keep = 2 * (step + 1) ** 2 * weight.detach().double(), weight.grad
        held.append(keep)  # (so that the next is somewhere else)
        lst = binding.make_grad_list([weight.grad])
        binding.sparsp_grad_squares(lst, ws)
        binding.sparsp_grad_clip(lst, 1.0, norm, ws)
        exact = float(want.norm())
        assert abs(float(norm) - exact) <= 20 * 2.0 ** -24 * exact
        assert bool(((keep.double() - want / (exact + 1e-6)).abs() <= 24 * 2.0 ** -24 * want.abs() / exact).all())
    assert len({h.data_ptr() for h in held}) == 5


@pytest.mark.gpu
@pytest.mark.parametrize("over", [False, True])
def test_a_large_list_in_place(over):
    """Matrices as a layer has them, written where they are."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    ts = [torch.empty(n, dtype=torch.bfloat16, device="cuda").normal_(0.0, 1.0, generator=gen) for n in (30_000_001, 12_345_678, 5)]
    keep = [t.clone() for t in ts]
    lst, ws, norm = binding.make_grad_list(ts), binding.make_grad_workspace(), torch.empty(1, device="cuda")
    exact = sum(float(t.double().square().sum()) for t in ts) ** 0.5
    limit = exact / 8 if over else 2 * exact
    binding.sparsp_grad_squares(lst, ws)
    binding.sparsp_grad_clip(lst, limit, norm, ws)
    assert abs(float(norm) - exact) <= 18 * 2.0 ** -24 * exact
    for t, k in zip(ts, keep):
        if not over:
            assert torch.equal(t, k)
        else:
            want = k.double() * (limit / (exact + 1e-6))
            assert bool(((t.double() - want).abs() <= (2.0 ** -8 + 2.0 ** -16) * want.abs()).all())
