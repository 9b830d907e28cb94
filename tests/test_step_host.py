"""Host side of the residual step and of lists of gradients: sizes, and what the calls refuse before anything is
launched."""
import math

import pytest
import torch

from paper_2609_32197_b200 import binding
from test_layer_host import At, INVALID, UNSUPPORTED, no_stream, refused  # noqa: F401


def pointers(names, base=1 << 20):
    return {k: At(base * (i + 1)) for i, k in enumerate(names)}


FWD = ["X", "Y", "gate", "wy", "by", "wr", "br", "R", "N", "sy", "sr"]
BWD = ["dN", "dR", "R", "Y", "gate", "wy", "by", "wr", "sy", "sr", "dX", "dY", "dgate", "dwy", "dby", "dwr", "dbr", "ws"]


def fwd(step, change):
    p = {**pointers(FWD), **change}
    return (binding.sparsp_gated_norm_fwd, step, *(p[k] for k in FWD))


def bwd(step, change):
    p = {**pointers(BWD), **change}
    return (binding.sparsp_gated_norm_bwd, step, *(p[k] for k in BWD))


@pytest.mark.parametrize("code,change", [
    (INVALID, {"dtype": 3}), (INVALID, {"weight_dtype": 1}), (INVALID, {"norm_y": 3}), (INVALID, {"norm_r": -1}),
    (INVALID, {"rows": -1}), (INVALID, {"rows_per_group": -1}), (INVALID, {"dim": 0}), (UNSUPPORTED, {"dim": 60}),
    (UNSUPPORTED, {"dim": 8200, "stride_x": 8200, "stride_y": 8200, "stride_n": 8200}), (INVALID, {"stride_x": 56}),
    (INVALID, {"stride_y": 68}), (INVALID, {"stride_n": 0}), (INVALID, {"eps": -1.0}), (INVALID, {"eps": math.inf}),
    (INVALID, {"eps": math.nan}), (UNSUPPORTED, {"rows": 1 << 38})])
def test_refused_steps(code, change):
    step = binding.make_gated_norm(4, 64, 0, "rms", "layer")
    for k, v in change.items():
        setattr(step, k, v)
    refused(code, binding.sparsp_gated_norm_workspace_bytes, step)
    refused(code, *fwd(step, {}))
    refused(code, *bwd(step, {}))


@pytest.mark.parametrize("norm_y,norm_r", [("none", "layer"), ("rms", "none")])
def test_what_belongs_to_an_absent_norm_is_refused(norm_y, norm_r):
    step = binding.make_gated_norm(4, 64, 0, norm_y, norm_r)
    gone = ["wy", "by", "sy"] if norm_y == "none" else ["wr", "br", "sr", "N"]
    for k in gone:
        refused(INVALID, *fwd(step, {q: None for q in gone if q != k}))
    gone = ["wy", "by", "sy", "dwy", "dby"] if norm_y == "none" else ["dN", "R", "wr", "sr", "dwr", "dbr"]
    for k in gone:
        refused(INVALID, *bwd(step, {q: None for q in gone if q != k}))


def test_refused_pointers():
    step = binding.make_gated_norm(4, 64, 0, "rms", "layer", stride_y=72)
    for k in FWD:
        refused(INVALID, *fwd(step, {k: At((1 << 20) + 4)}))
    for k in ("X", "Y", "R", "N"):
        refused(INVALID, *fwd(step, {k: None}))
    p = pointers(FWD)
    for a, b in (("R", "Y"), ("N", "X"), ("R", "N"), ("N", "Y"), ("R", "gate"), ("N", "wr"), ("sy", "sr"), ("sr", "br")):
        refused(INVALID, *fwd(step, {a: p[b]}))  # (N at Y: the strides differ)
    for k in BWD:
        refused(INVALID, *bwd(step, {k: At((1 << 20) + 4)}))
    for k in ("dN", "R", "Y", "sy", "sr", "ws"):
        refused(INVALID, *bwd(step, {k: None}))
    p = pointers(BWD)
    for a, b in (("dX", "dN"), ("dX", "R"), ("dX", "Y"), ("dX", "dY"), ("dY", "dR"), ("dY", "Y"), ("dgate", "gate"),
                 ("dwr", "dbr"), ("dwy", "wy")):
        refused(INVALID, *bwd(step, {a: p[b]}))
    refused(INVALID, *bwd(binding.make_gated_norm(4, 64, 0, "none", "none"),
                          {k: None for k in ("dN", "dR", "R", "wy", "by", "wr", "sy", "sr", "dwy", "dby", "dwr", "dbr")}))


def test_step_workspace_of_more_rows_serves_fewer():
    for dim in (8, 512, 1928, 5120, 8192):
        for dtype in (torch.bfloat16, torch.float32):
            size = [binding.sparsp_gated_norm_workspace_bytes(binding.make_gated_norm(r, dim, per, dtype=dtype))
                    for r in (0, 1, 2, 100, 5000, 1 << 20) for per in (0,)]
            assert size == sorted(size) and size[0] >= 256


def grads(*parts, outs=None, dtype=torch.bfloat16):
    """parts: (address, size)"""
    import ctypes
    n = len(parts)
    a, s = (ctypes.c_void_p * n)(*(p[0] for p in parts)), (ctypes.c_int64 * n)(*(p[1] for p in parts))
    o = None if outs is None else (ctypes.c_void_p * n)(*outs)
    lst = binding.sparsp_grad_list(n, binding.DTYPES[dtype], ctypes.addressof(a), None if o is None else ctypes.addressof(o),
                                   ctypes.addressof(s))
    lst.kept = (a, s, o)
    return lst


def test_refused_lists():
    ws = At(1 << 20)
    for bad in (grads((4096, -1)), grads((0, 8)), grads((4097, 8)), grads((4098, 8), dtype=torch.float32),
                grads((4096, 8), outs=[None]), grads((4096, 8), outs=[8193]), grads((4096, 1 << 41))):
        refused(INVALID, binding.sparsp_grad_squares, bad, ws)
        refused(INVALID, binding.sparsp_grad_clip, bad, 1.0, None, ws)
    good = grads((4096, 8), (8192, 8))
    for change in ({"dtype": 3}, {"count": -1}, {"grads": None}, {"sizes": None}):
        lst = grads((4096, 8), (8192, 8))
        for k, v in change.items():
            setattr(lst, k, v)
        refused(INVALID, binding.sparsp_grad_squares, lst, ws)
        refused(INVALID, binding.sparsp_grad_clip, lst, 1.0, None, ws)
    for limit in (0.0, -1.0, math.nan):
        refused(INVALID, binding.sparsp_grad_clip, good, limit, None, ws)
    for bad in (None, At((1 << 20) + 16)):
        refused(INVALID, binding.sparsp_grad_squares, good, bad)
        refused(INVALID, binding.sparsp_grad_clip, good, 1.0, None, bad)
    refused(INVALID, binding.sparsp_grad_clip, good, 1.0, At(4098), ws)


def test_gradients_that_overlap_are_not_clipped():
    ws = At(1 << 20)
    for bad in (grads((8192, 8), (8192, 8)), grads((8192, 8), (8200, 8)), grads((8192, 8), (4096, 2049)),
                grads((4096, 8), (8192, 8), outs=[65536, 65536])):
        refused(INVALID, binding.sparsp_grad_clip, bad, 1.0, None, ws)


def test_make_grad_list():
    a, b = torch.zeros(4), torch.zeros(6)
    lst = binding.make_grad_list([a, b])
    assert (lst.count, lst.dtype) == (2, binding.SPARSP_FP32)
    assert binding.make_grad_list([]).count == 0
    for bad in (([a, b.double()],), ([a, b.half()],), ([b.view(2, 3).T],), ([a], [b]), ([a, b], [a]), ([a], [a.half()])):
        with pytest.raises(ValueError):
            binding.make_grad_list(*bad)
