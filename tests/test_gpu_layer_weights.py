"""A layer with projections in 4 bits goes on with its weights as they are changed."""
import pytest
import torch

import fp4_reference as fp4
from paper_2609_32197_b200 import binding, dit_layer
from test_gpu_dit_layer import off
from test_gpu_gated_layer import check_projection, make

pytestmark = pytest.mark.gpu
GRID = ((3, 10, 17), 45, 3, 64, 352)


def exponent_of(fmt):
    return -4 if fmt == "nvfp4" else 0


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
def test_a_training_step_sees_the_weight_as_it_is(fmt):
    layer, x, dy = make(*GRID, fmt)
    layer.forward(x)
    layer.training_step(x, dy)
    layer.w_down.mul_(-0.5).add_(0.01)
    grads = {k: v.clone() for k, v in layer.training_step(x, dy).items()}
    linear = layer.fp4["down"]
    check_projection(layer.h, linear, layer.w_down, fmt, exponent_of(fmt), layer.f)
    values = fp4.quantize(layer.w_down, fmt, linear.described.exponent)[2]
    assert torch.equal(linear.values.double(), values.to(torch.bfloat16).double())
    other, _, _ = make(*GRID, fmt)
    other.a.copy_(layer.a)
    other.w_down.copy_(layer.w_down)
    other.update_weights()
    want = other.training_step(x, dy)
    assert all(off(grads[k], want[k]) <= 0.02 for k in want)
    assert layer.status() == binding.SPARSP_OK


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
def test_a_forward_pass_after_new_weights(fmt):
    """All of them are taken anew, with the exponents that they need now."""
    layer, x, _ = make(*GRID, fmt)
    layer.forward(x)
    for w in (layer.w_qkv, layer.w_out, layer.w_down):
        w.mul_(37.0)
    layer.update_weights()
    y = layer.forward(x)
    if fmt == "nvfp4":
        most, e = float(layer.w_down.abs().max()), layer.fp4["down"].described.exponent
        assert 2688 * 2.0 ** (e - 1) < most <= 2688 * 2.0 ** e
    e = exponent_of(fmt)
    check_projection(layer.n, layer.fp4["qkv2"], layer.w_qkv[2 * layer.width:], fmt, e, layer.qkv[2])
    check_projection(layer.o, layer.fp4["out"], layer.w_out, fmt, e, layer.a)
    check_projection(layer.h, layer.fp4["down"], layer.w_down, fmt, e, layer.f)
    fresh, _, _ = make(*GRID, fmt)
    for name in ("w_qkv", "w_out", "w_down"):
        getattr(fresh, name).copy_(getattr(layer, name))
    fresh.update_weights()
    assert torch.equal(fresh.forward(x), y)
    assert layer.status() == binding.SPARSP_OK


def test_new_weights_under_a_kept_exponent():
    """Without a question to the device, so that it can be captured: values beyond what the exponent holds become its largest."""
    layer, _, _ = make(*GRID, "nvfp4")
    linear = layer.fp4["down"]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        linear.requantize(keep_exponent=True)
    layer.w_down.mul_(0.7)
    layer.w_down[3, 5] = 2.0 ** 20
    graph.replay()
    want = fp4.quantize(layer.w_down, "nvfp4", linear.described.exponent)[2]
    assert torch.equal(linear.values.double(), want.to(torch.bfloat16).double())
    assert float(linear.values[3, 5]) == 6 * 448 * 2.0 ** linear.described.exponent


@pytest.mark.parametrize("most", [0.0, 2.0 ** -70, 1.0, 2688.0, 2689.0])
def test_the_exponent_of_a_weight(most):
    """The least with which the largest value is not cut off, unless that is too small to matter."""
    w = torch.zeros(64, 64, device="cuda")
    w[1, 1], w[2, 2] = most, 1e-25
    linear = dit_layer.Fp4Linear(w, 4, "nvfp4")
    e = linear.described.exponent
    if most >= 1.0:
        assert 2688 * 2.0 ** (e - 1) < most <= 2688 * 2.0 ** e
    want = fp4.quantize(w, "nvfp4", e)[2].float()
    assert torch.equal(linear.values, want)
