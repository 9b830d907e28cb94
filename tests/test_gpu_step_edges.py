"""Calls at the edges of the operators between a layer's products: tensors beyond 2^31 elements, calls on two streams at
once, calls one behind the other on one workspace, captured calls on new values."""
import pytest
import torch

from paper_2609_32197_b200 import binding

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def normal(seed, *dims, dtype=BF, scale=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(dims, dtype=dtype, device="cuda").normal_(0.0, scale, generator=gen)


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
def test_quantize_beyond_32_bits(fmt):
    rows, cols = 520000 + 5, 4160
    x = normal(1, rows, cols)
    fp4 = binding.make_fp4(rows, cols, fmt)
    codes, scales = binding.make_fp4_operand(fp4)
    binding.sparsp_fp4_quantize(fp4, x, codes, scales, x)
    first = rows // 128 * 128 - 128  # the last whole group of 128 rows and what lies behind it
    tail = normal(1, rows, cols)[first:].clone()
    small = binding.make_fp4(rows - first, cols, fmt)
    c, s = binding.make_fp4_operand(small)
    binding.sparsp_fp4_quantize(small, tail, c, s, tail)
    assert torch.equal(codes[first:], c) and torch.equal(x[first:], tail)
    assert torch.equal(scales[-s.numel():], s)


def test_product_beyond_32_bits():
    rows, cols, depth = 524288 + 300, 4104, 64
    a, b = normal(2, rows, depth), normal(3, cols, depth)
    qa, qb = (binding.make_fp4(m.shape[0], depth) for m in (a, b))
    oa, ob = binding.make_fp4_operand(qa), binding.make_fp4_operand(qb)
    binding.sparsp_fp4_quantize(qa, a, *oa, None)
    binding.sparsp_fp4_quantize(qb, b, *ob, None)
    d = binding.make_fp4_product(rows, cols, depth)
    c, ws = torch.empty(rows, cols, dtype=BF, device="cuda"), binding.make_fp4_product_workspace(d)
    binding.sparsp_fp4_product(d, *oa, *ob, None, c, ws)
    first = rows // 128 * 128 - 256
    tail = binding.make_fp4(rows - first, depth)
    ot = binding.make_fp4_operand(tail)
    binding.sparsp_fp4_quantize(tail, a[first:].clone(), *ot, None)
    dt = binding.make_fp4_product(rows - first, cols, depth)
    want = torch.empty(rows - first, cols, dtype=BF, device="cuda")
    binding.sparsp_fp4_product(dt, *ot, *ob, None, want, binding.make_fp4_product_workspace(dt))
    assert torch.equal(c[first:], want)
    assert binding.sparsp_status(ws) == binding.SPARSP_OK


def test_residual_step_beyond_32_bits():
    rows, dim = 530000, 4096
    x, y = normal(4, rows, dim), normal(5, rows, dim)
    gate, wr, br = (normal(6 + i, 1, dim, dtype=torch.float32) for i in range(3))
    last = slice(rows - 100, rows)
    xt, yt = x[last].clone(), y[last].clone()
    step, small = (binding.make_gated_norm(n, dim, weight_dtype=torch.float32) for n in (rows, 100))
    sr, st = torch.empty(rows, 2, device="cuda"), torch.empty(100, 2, device="cuda")
    binding.sparsp_gated_norm_fwd(step, x, y, gate, None, None, wr, br, x, y, None, sr)  # in place: r and n
    binding.sparsp_gated_norm_fwd(small, xt, yt, gate, None, None, wr, br, xt, yt, None, st)
    assert torch.equal(x[last], xt) and torch.equal(y[last], yt) and torch.equal(sr[last], st)
    dr = normal(9, rows, dim)
    dy, ws = torch.empty_like(x), binding.make_gated_norm_workspace(step)
    dt, dyt = dr[last].clone(), torch.empty_like(xt)
    binding.sparsp_gated_norm_bwd(step, y, dr, x, y, gate, None, None, wr, None, sr, dr, dy, None, None, None, None, None, ws)
    binding.sparsp_gated_norm_bwd(small, yt, dt, xt, yt, gate, None, None, wr, None, st, dt, dyt, None, None, None, None, None,
                                  binding.make_gated_norm_workspace(small))
    assert torch.equal(dr[last], dt) and torch.equal(dy[last], dyt)


def test_clip_beyond_32_bits():
    n = (1 << 31) + 12345
    g = torch.full((n,), 2.0 ** -10, dtype=BF, device="cuda")
    g[-1] = 3.0
    lst, ws, norm = binding.make_grad_list([g, torch.ones(5, dtype=BF, device="cuda")]), binding.make_grad_workspace(), torch.empty(
        1, device="cuda")
    binding.sparsp_grad_squares(lst, ws)
    want = ((n - 1) * 2.0 ** -20 + 9.0 + 5.0) ** 0.5
    binding.sparsp_grad_clip(lst, want / 4, norm, ws)
    assert abs(float(norm) - want) <= 2.0 ** -19 * want
    assert float(g[-1]) == 0.75 and float(g[0]) == 2.0 ** -12 and bool((g[:-1] == 2.0 ** -12).all())


def product_of(seed, m, n, k, fmt):
    a, b = normal(seed, m, k), normal(seed + 1, n, k, scale=k ** -0.5)
    ops = []
    for x in (a, b):
        q = binding.make_fp4(x.shape[0], k, fmt)
        ops += binding.make_fp4_operand(q)
        binding.sparsp_fp4_quantize(q, x, *ops[-2:], None)
    d = binding.make_fp4_product(m, n, k, fmt)
    return d, ops, torch.empty(m, n, dtype=BF, device="cuda"), binding.make_fp4_product_workspace(d)


def test_two_streams_at_once():
    """Products, steps and clippings on two streams, each with its own workspace, as on one."""
    jobs = [product_of(20, 1, 10240, 2048, "nvfp4"), product_of(22, 70, 1280, 4096, "mxfp4"), product_of(24, 700, 2568, 1056, "nvfp4"),
            product_of(26, 1500, 520, 2048, "mxfp4")]
    grads = [normal(30 + i, 300001, dtype=torch.float32) for i in range(2)]
    lists = [binding.make_grad_list([g], [torch.empty_like(g)]) for g in grads]
    works, norms = [binding.make_grad_workspace() for _ in range(2)], [torch.empty(1, device="cuda") for _ in range(2)]

    def run(i):
        for d, ops, c, ws in jobs[i::2]:
            binding.sparsp_fp4_product(d, *ops, None, c, ws)
        binding.sparsp_grad_squares(lists[i], works[i])
        binding.sparsp_grad_clip(lists[i], 1.0, norms[i], works[i])

    for i in range(2):
        run(i)
    want = [c.clone() for _, _, c, _ in jobs] + [n.clone() for n in norms] + [lst.kept[1][0].clone() for lst in lists]
    for _, _, c, _ in jobs:
        c.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                run(i)
    torch.cuda.synchronize()
    got = [c for _, _, c, _ in jobs] + norms + [lst.kept[1][0] for lst in lists]
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_one_workspace_for_calls_of_every_size():
    jobs = [product_of(40 + 2 * i, m, n, k, "nvfp4") for i, (m, n, k) in enumerate(
        [(1, 512, 2048), (128, 256, 4096), (300, 1000, 512), (5, 20480, 512), (17, 128, 256)])]
    ws = binding.make_fp4_product_workspace(binding.make_fp4_product(1 << 17, 1 << 17, 1 << 17))
    want = []
    for d, ops, c, own in jobs:
        binding.sparsp_fp4_product(d, *ops, None, c, own)
        want.append(c.clone())
    for _ in range(3):
        for (d, ops, c, _), w in zip(jobs, want):
            c.zero_()
            binding.sparsp_fp4_product(d, *ops, None, c, ws)
            assert torch.equal(c, w)
    assert binding.sparsp_status(ws) == binding.SPARSP_OK
    step = binding.make_gated_norm(5000, 1032, 70)
    big = binding.make_gated_norm_workspace(step)
    for rows, per in ((5000, 70), (3, 0), (148, 1), (1, 1), (4999, 2500)):
        y, dr, gate = normal(60, rows, 1032), normal(61, rows, 1032), normal(62, -(-rows // (per or rows)), 1032)
        s = binding.make_gated_norm(rows, 1032, per, norm_r="none")
        out = []
        for ws in (binding.make_gated_norm_workspace(s), big):
            dy, dgate = torch.empty_like(y), torch.empty_like(gate)
            binding.sparsp_gated_norm_bwd(s, None, dr, None, y, gate, None, None, None, None, None, None, dy, dgate, None, None,
                                          None, None, ws)
            out.append((dy, dgate))
        assert all(torch.equal(a, b) for a, b in zip(*out))
