"""The gated layer: the residual steps, the projections in 4 bits and the clipped gradients as they are used together.

In bf16 against the same layer in plain torch operations in 64 bits, with the bound of the layer without gates (2 %: about
ten roundings of 2^-9 / sqrt 3 each).  In 4 bits a rounding that differs moves a value by a step, so each projection is
compared on the input that it was given."""
import pytest
import torch

import fp4_reference as fp4
from layer_reference import TINY, UNIT, activation, close, layer_norm
from paper_2609_32197_b200 import binding, dit_layer, synth
from test_gpu_dit_layer import off, plain_attention_half

pytestmark = pytest.mark.gpu
EPS = 1e-5


def make(grid, n_text, heads, head_dim, hidden, projections="bf16"):
    wl = synth.Workload("layer", heads, head_dim, grid, n_text, 64, 4, None, 1)
    layer = dit_layer.GatedDitLayer(wl, hidden, projections=projections)
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, dy = (torch.empty(wl.n_tokens, layer.width, dtype=torch.bfloat16, device="cuda").normal_(0.0, 1.0, generator=gen)
             for _ in range(2))
    return layer, x, dy


def plain_behind(x, a, w):
    x1 = x + w["gate1"] * a
    m, _, _ = layer_norm(x1, w["scale2"], w["shift2"], EPS, x1.shape[0])
    return x1 + w["gate2"] * (activation("silu", m @ w["w_gate"].T)[0] * (m @ w["w_up"].T) @ w["w_down"].T)


NAMES = ("gate1", "gate2", "scale2", "shift2", "w_gate", "w_up", "w_down")


@pytest.mark.parametrize("grid,n_text,heads,head_dim,hidden", [((4, 12, 16), 0, 3, 64, 512), ((3, 10, 17), 45, 2, 128, 328)])
def test_a_gated_layer(grid, n_text, heads, head_dim, hidden):
    layer, x, _ = make(grid, n_text, heads, head_dim, hidden)
    y = layer.forward(x)
    assert off(layer.a, plain_attention_half(layer, x)) <= 0.02
    w = {k: getattr(layer, k).double() for k in NAMES}
    assert off(y.double() - x.double(), plain_behind(x.double(), layer.a.double(), w) - x.double()) <= 0.02
    assert torch.equal(layer.forward(x), y)
    assert layer.status() == binding.SPARSP_OK


@pytest.mark.parametrize("share", [0.25, 4.0])
def test_a_training_step(share):
    layer, x, dy = make((3, 10, 11), 21, 4, 64, 616)
    layer.attention(x)
    layer.project_out()
    whole = {k: v.clone() for k, v in layer.training_step(x, dy).items()}
    norm = float(layer.grad_norm)
    leaves = {k: getattr(layer, k).double().requires_grad_() for k in NAMES}
    X, A = x.double().requires_grad_(), layer.a.double().requires_grad_()
    with torch.enable_grad():
        plain_behind(X, A, leaves).backward(dy.double())
    want = {**{k: v.grad for k, v in leaves.items()}, "x": X.grad, "a": A.grad}
    for k in want:
        assert off(whole[k], want[k]) <= 0.02, k
    exact = float(sum(whole[k].double().square().sum() for k in NAMES)) ** 0.5
    assert abs(norm - exact) <= 1e-6 * exact
    clipped = layer.training_step(x, dy, share * norm)
    assert float(layer.grad_norm) == norm
    factor = min(1.0, share * norm / (norm + 1e-6))
    for k in NAMES:
        t = whole[k].dtype
        want_k = whole[k].double() * factor
        close(clipped[k], want_k, (UNIT[t] + 1e-6) * want_k.abs() + TINY[t], k)
    for k in ("x", "a"):
        assert torch.equal(clipped[k], whole[k])
    assert layer.status() == binding.SPARSP_OK


def check_projection(x, linear, weight, fmt, exponent, out):
    ew = linear.described.exponent
    a, b = fp4.quantize(x, fmt, exponent)[2], fp4.quantize(weight, fmt, ew)[2]
    want = a @ b.T
    bound = (x.shape[1] / 16 + 8) * 2.0 ** -23 * (a.abs() @ b.abs().T)
    close(out, want, bound + UNIT[out.dtype] * (want.abs() + bound) + TINY[out.dtype], "projection")


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
def test_projections_in_4_bits(fmt):
    layer, x, dy = make((3, 10, 17), 45, 3, 64, 352, fmt)
    y = layer.forward(x)
    e = -4 if fmt == "nvfp4" else 0
    check_projection(layer.n, layer.fp4["qkv2"], layer.w_qkv[2 * layer.width:], fmt, e, layer.qkv[2])  # (q and k are turned)
    check_projection(layer.o, layer.fp4["out"], layer.w_out, fmt, e, layer.a)
    check_projection(layer.h, layer.fp4["down"], layer.w_down, fmt, e, layer.f)
    want = layer.x1.double() + layer.gate2.double() * layer.f.double()
    close(y, want, 2.0 ** -22 * (layer.x1.double().abs() + want.abs()) + UNIT[y.dtype] * want.abs(), "y")
    grads = layer.training_step(x, dy, 1.0)
    values = fp4.quantize(layer.h, fmt, e)[2]
    assert torch.equal(layer.h_values.double(), values.to(torch.bfloat16).double())
    df = dy.double() * layer.gate2.double()
    scale = min(1.0, 1.0 / (float(layer.grad_norm) + 1e-6))
    assert off(grads["w_down"], df.T @ values * scale) <= 0.02
    assert all(bool(g.isfinite().all()) for g in grads.values())
    assert layer.status() == binding.SPARSP_OK


def test_a_layer_in_a_graph_beside_an_eager_one():
    """Captured once, replayed on new input, while another layer's eager step lives."""
    layer, x, dy = make((3, 10, 11), 21, 2, 64, 288, "nvfp4")
    other, _, _ = make((3, 10, 11), 21, 2, 64, 288)
    layer.forward(x)
    eager = {k: v.clone() for k, v in other.training_step(x, dy, 1.0).items()}
    graph = torch.cuda.CUDAGraph()
    held = x.clone()
    with torch.cuda.graph(graph):
        y = layer.forward(held)
        grads = layer.training_step(held, dy, 1.0)
    fresh = torch.randn_like(x)
    held.copy_(fresh)
    graph.replay()
    got_y, got = y.clone(), {k: v.clone() for k, v in grads.items()}
    assert torch.equal(layer.forward(fresh), got_y)
    want = layer.training_step(fresh, dy, 1.0)
    for k in want:
        assert torch.equal(want[k], got[k]), k
    again = other.training_step(x, dy, 1.0)
    for k in eager:
        assert torch.equal(eager[k], again[k]), k
