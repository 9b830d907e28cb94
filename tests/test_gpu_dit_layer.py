"""The layer example: every call together, against the same layer in plain torch operations in 64 bits.

The layer rounds to bf16 at about ten places between its input and what each half adds to it; each rounding is 2^-9 / sqrt 3
of its values at most in the root mean square and the products between them keep relative errors, so a half's addition is
off by about sqrt(10) 2^-9 / sqrt 3 = 0.4 % in the norm; gradients by as much again.  The bound is 2 %."""
import pytest
import torch

from layer_reference import activation, layer_norm, layer_norm_back
from paper_2609_32197_b200 import binding, dit_layer, synth

pytestmark = pytest.mark.gpu
EPS = 1e-5


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


def plain_attention_half(layer, x):
    wl, D = layer.wl, layer.width
    H, d, N = wl.heads, wl.head_dim, wl.n_tokens
    n, _, _ = layer_norm(x.double(), layer.scale1.double(), layer.shift1.double(), EPS, N)
    q, k, v = ((n @ layer.w_qkv[i * D:(i + 1) * D].double().T).view(N, H, d).transpose(0, 1) for i in range(3))
    t, h, w = torch.meshgrid(*(torch.arange(g, device="cuda", dtype=torch.float64) for g in wl.grid), indexing="ij")
    pairs = dit_layer.axis_pairs(d)
    angle = torch.cat([p.reshape(-1, 1) * 10000.0 ** (-torch.arange(m, device="cuda", dtype=torch.float64) / m)
                       for p, m in zip((t, h, w), pairs)], 1)
    angle = torch.cat((angle, torch.zeros(wl.n_text, angle.shape[1], device="cuda", dtype=torch.float64)))
    turn = torch.polar(torch.ones_like(angle), angle)
    q, k = (torch.view_as_real(torch.view_as_complex(z.reshape(H, N, d // 2, 2)) * turn).reshape(H, N, d) for z in (q, k))
    words = layer.mask[0].to(torch.int64) & 0xffffffff
    bits = (words[..., None] >> torch.arange(32, device="cuda")) & 1
    kept = bits.reshape(H, words.shape[1], -1).bool()[:, :, :-(-N // wl.block)]
    kept = kept.repeat_interleave(wl.block, 1).repeat_interleave(wl.block, 2)[:, :N, :N]
    score = (q @ k.transpose(1, 2)) * d ** -0.5
    o = torch.softmax(score.masked_fill(~kept, -float("inf")), -1) @ v
    return o.transpose(0, 1).reshape(N, D) @ layer.w_out.double().T


def plain_feed_forward_half(layer, x1, w):
    m, mean, rstd = layer_norm(x1, w["scale2"], w["shift2"], EPS, x1.shape[0])
    return activation("silu", m @ w["w_gate"].T)[0] * (m @ w["w_up"].T) @ w["w_down"].T


@pytest.mark.parametrize("grid,n_text,heads,head_dim,hidden", [((4, 12, 16), 0, 3, 64, 512), ((3, 10, 17), 45, 2, 128, 328)])
def test_a_layer(grid, n_text, heads, head_dim, hidden):
    wl = synth.Workload("layer", heads, head_dim, grid, n_text, 64, 4, None, 1)
    layer = dit_layer.DitLayer(wl, hidden)
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.empty(wl.n_tokens, layer.width, dtype=torch.bfloat16, device="cuda").normal_(0.0, 1.0, generator=gen)
    x1 = layer.attention_half(x)
    assert off(x1.double() - x.double(), plain_attention_half(layer, x)) <= 0.02
    w = {k: getattr(layer, k).double() for k in ("scale2", "shift2", "w_gate", "w_up", "w_down")}
    y = layer.feed_forward_half(x1)
    assert off(y.double() - x1.double(), plain_feed_forward_half(layer, x1.double(), w)) <= 0.02
    assert torch.equal(layer.forward(x), y)
    assert layer.status() == binding.SPARSP_OK


def test_a_training_step_of_the_feed_forward_half():
    wl = synth.Workload("layer", 4, 64, (3, 10, 11), 21, 64, 3, None, 1)
    layer = dit_layer.DitLayer(wl, 616)
    gen = torch.Generator(device="cuda").manual_seed(4)
    x1, dy = (torch.empty(wl.n_tokens, layer.width, dtype=torch.bfloat16, device="cuda").normal_(0.0, 1.0, generator=gen)
              for _ in range(2))
    assert torch.equal(layer.feed_forward_half(x1, training=True), layer.feed_forward_half(x1))
    layer.feed_forward_half(x1, training=True)
    got = layer.feed_forward_backward(x1, dy)
    with torch.enable_grad():
        w = {k: getattr(layer, k).double().requires_grad_() for k in ("scale2", "shift2", "w_gate", "w_up", "w_down")}
        x = x1.double().requires_grad_()
        loss = ((x + plain_feed_forward_half(layer, x, w)) * dy.double()).sum()
        want = dict(zip(["x", *w], torch.autograd.grad(loss, [x, *w.values()])))
    for name, grad in want.items():
        assert off(got[name], grad) <= 0.02, name
    assert layer.status() == binding.SPARSP_OK


def test_the_layer_in_a_graph():
    """Forward and the training step are stream-ordered work: captured once, replayed on new inputs in the same buffers."""
    wl = synth.WORKLOADS["tiny"]
    layer = dit_layer.DitLayer(wl, 512)
    x = torch.empty(wl.n_tokens, layer.width, dtype=torch.bfloat16, device="cuda").normal_(0.0, 1.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            y = layer.forward(x)
            layer.feed_forward_half(x, training=True)
            grads = layer.feed_forward_backward(x, x)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = layer.forward(x)
        layer.feed_forward_half(x, training=True)
        grads = layer.feed_forward_backward(x, x)
    x.normal_(0.0, 1.0)
    graph.replay()
    torch.cuda.synchronize()
    got = [y.clone()] + [grads[k].clone() for k in sorted(grads)]
    want_y = layer.forward(x)
    layer.feed_forward_half(x, training=True)
    want = layer.feed_forward_backward(x, x)
    assert all(torch.equal(a, b) for a, b in zip(got, [want_y] + [want[k] for k in sorted(want)]))
