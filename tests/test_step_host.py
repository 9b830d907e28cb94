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
                                   ctypes.addressof(s), 0, 0, 0)
    lst.kept = (a, s, o)
    return lst


def table_of(lst):
    return torch.zeros(binding.sparsp_grad_table_bytes(lst), dtype=torch.uint8)


def test_refused_lists():
    room = torch.zeros(1 << 16, dtype=torch.uint8)
    bad = [grads((4096, -1)), grads((0, 8)), grads((4097, 8)), grads((4098, 8), dtype=torch.float32),
           grads((4096, 8), outs=[None]), grads((4096, 8), outs=[8193]), grads((4096, 1 << 41))]
    for change in ({"dtype": 3}, {"count": -1}, {"grads": None}, {"sizes": None}):
        bad.append(grads((4096, 8), (8192, 8)))
        for k, v in change.items():
            setattr(bad[-1], k, v)
    for lst in bad:
        refused(INVALID, binding.sparsp_grad_table_bytes, lst)
        refused(INVALID, binding.sparsp_grad_table, lst, room)
    good = grads((4096, 8), (8192, 8))
    refused(INVALID, binding.sparsp_grad_table, good, None)
    refused(INVALID, binding.sparsp_grad_table, good, At(4104))


def test_refused_calls():
    ws = At(1 << 20)
    lst = grads((4096, 8), (8192, 8))
    lst.table = At(1 << 16)
    refused(INVALID, binding.sparsp_grad_squares, lst, ws)  # no table yet
    refused(INVALID, binding.sparsp_grad_clip, lst, 1.0, None, ws)
    binding.sparsp_grad_table(lst, table_of(lst))
    assert (lst.chunks, lst.ctas, lst.in_place) == (2, 2, 1)
    for limit in (0.0, -1.0, math.nan):
        refused(INVALID, binding.sparsp_grad_clip, lst, limit, None, ws)
    for bad in (None, At((1 << 20) + 16)):
        refused(INVALID, binding.sparsp_grad_squares, lst, bad)
        refused(INVALID, binding.sparsp_grad_clip, lst, 1.0, None, bad)
    refused(INVALID, binding.sparsp_grad_clip, lst, 1.0, At(4098), ws)
    for bad in (None, At(4104)):
        lst.table = bad
        refused(INVALID, binding.sparsp_grad_squares, lst, ws)
        refused(INVALID, binding.sparsp_grad_clip, lst, 1.0, None, ws)


def test_gradients_that_overlap_are_refused():
    for bad in (grads((8192, 8), (8192, 8)), grads((8192, 8), (8200, 8)), grads((8192, 8), (4096, 2049)),
                grads((4096, 8), (8192, 8), outs=[65536, 65536])):
        refused(INVALID, binding.sparsp_grad_table, bad, table_of(bad))


@pytest.mark.parametrize("count,dtype", [(0, torch.bfloat16), (1, torch.bfloat16), (700, torch.float32), (3000, torch.float16)])
def test_table(count, dtype):
    """Every chunk of every tensor belongs to the run of one CTA, which knows the tensor that it begins in."""
    import random
    rng = random.Random(count)
    e = 4 if dtype == torch.float32 else 2
    parts, at = [], 1 << 20
    for _ in range(count):
        size = rng.choice((0, 1, 7, 4095, 4096, 4097, 8192, 8193, 50000))
        at += rng.choice((0, e, 16))
        parts.append((at, size))
        at += size * e
    lst = grads(*parts, dtype=dtype)
    table = table_of(lst)
    binding.sparsp_grad_table(lst, table)
    words = table[:(count + 1) * 32].view(torch.int64).view(-1, 4).tolist()
    begins = table[(count + 1) * 32:].view(torch.int32).tolist()
    each, chunk = 16384 // e, 0
    there = [p for p in parts if p[1] > 0]
    for (address, size), (source, to, n, first) in zip(there, words):
        assert (source, to, n, first) == (address, address, size, chunk)
        skip = min(-address % 16 // e, size)
        chunk += max(1, -(-(size - skip) // each))
    assert words[len(there)][3] == chunk == lst.chunks and lst.ctas == max(1, min(chunk, 8 * 148))
    firsts = [w[3] for w in words[:len(there) + 1]]
    q, r = divmod(chunk, lst.ctas)
    for b in range(lst.ctas + 1):
        begin, t = b * q + min(b, r), begins[b]
        assert t == len(there) if begin == chunk else firsts[t] <= begin < firsts[t + 1]


def test_make_grad_list():
    a, b = torch.zeros(4), torch.zeros(6)
    lst = binding.make_grad_list([a, b])
    assert (lst.count, lst.dtype) == (2, binding.SPARSP_FP32)
    for bad in (([a, b.double()],), ([a, b.half()],), ([b.view(2, 3).T],), ([a], [b]), ([a, b], [a]), ([a], [a.half()])):
        with pytest.raises(ValueError):
            binding.make_grad_list(*bad)
