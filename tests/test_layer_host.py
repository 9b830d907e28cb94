"""Host side of the token-wise operators: frequencies, sizes, and what the calls refuse before anything is launched."""
import math

import pytest
import torch

from paper_2609_32197_b200 import binding
from paper_2609_32197_b200.binding import SparspError

INVALID, UNSUPPORTED = binding.SPARSP_ERR_INVALID_ARG, binding.SPARSP_ERR_UNSUPPORTED


class At:
    """A tensor of this address, for arguments that are refused before anybody reads them."""

    def __init__(self, address=4096):
        self.address = address

    def data_ptr(self):
        return self.address

    def dim(self):
        return 2


@pytest.fixture(autouse=True)
def no_stream(monkeypatch):
    monkeypatch.setattr(binding, "_stream_handle", lambda: None)


def refused(code, call, *args):
    with pytest.raises(SparspError) as e:
        call(*args)
    assert e.value.code == code, str(e.value)


@pytest.mark.parametrize("n", [1, 2, 21, 64])
def test_frequencies(n):
    plain, one = binding.sparsp_rotary_frequencies(n, 10000.0)
    assert one == 1.0
    for i in range(n):
        assert math.isclose(plain[i], 10000.0 ** (-i / n), rel_tol=1e-14)
    linear, one = binding.sparsp_rotary_frequencies(n, 10000.0, "linear", 4.0)
    assert one == 1.0 and all(math.isclose(a, b / 4, rel_tol=1e-14) for a, b in zip(linear, plain))
    ntk, one = binding.sparsp_rotary_frequencies(n, 10000.0, "ntk", 8.0)
    assert one == 1.0 and ntk[0] == 1.0
    if n > 1:  # the slowest pair is stretched by the factor, the fastest is not
        assert math.isclose(ntk[n - 1], plain[n - 1] / 8, rel_tol=1e-12)
    yarn, amplitude = binding.sparsp_rotary_frequencies(n, 10000.0, "yarn", 4.0, 4096.0)
    assert math.isclose(amplitude, 0.1 * math.log(4.0) + 1.0)
    for i in range(n):
        assert plain[i] / 4 * (1 - 1e-14) <= yarn[i] <= plain[i] * (1 + 1e-14)
    if n == 64:
        turns = [4096 * float(f) / (2 * math.pi) for f in plain]
        low = math.floor(64 * math.log(4096 / (2 * math.pi * 32)) / math.log(10000.0))
        for i in range(n):
            if i <= low:
                assert turns[i] > 31 and math.isclose(yarn[i], plain[i], rel_tol=1e-14)
            if turns[i] < 0.85:
                assert math.isclose(yarn[i], plain[i] / 4, rel_tol=1e-14)


@pytest.mark.parametrize("n", [1, 3, 32, 64])
@pytest.mark.parametrize("original,theta,factor", [(4096.0, 10000.0, 4.0), (32768.0, 10000.0, 8.0), (65536.0, 10000.0, 4.0),
                                                   (262144.0, 10000.0, 2.0), (65536.0, 500000.0, 16.0)])
def test_yarn_of_every_pair(n, original, theta, factor):
    """As published, in rotated channels: a frequency is interpolated by how far its pair is between the channels that
    turn 32 times and once over the original length, those limited to 0 .. channels - 1."""
    channels = 2 * n
    turning = lambda times: channels * math.log(original / (times * 2 * math.pi)) / (2 * math.log(theta))  # noqa: E731
    low, high = max(math.floor(turning(32)), 0), min(math.ceil(turning(1)), channels - 1)
    if low == high:
        high += 0.001
    got, amplitude = binding.sparsp_rotary_frequencies(n, theta, "yarn", factor, original, 32.0, 1.0)
    for i in range(n):
        extrapolated = 1.0 / theta ** (2 * i / channels)
        ramp = min(max((i - low) / (high - low), 0.0), 1.0)
        want = extrapolated / factor * ramp + extrapolated * (1.0 - ramp)
        assert math.isclose(got[i], want, rel_tol=1e-13), (i, low, high)
    assert math.isclose(amplitude, 0.1 * math.log(factor) + 1.0, rel_tol=1e-15)


def test_frequencies_refused():
    f = binding.sparsp_rotary_frequencies
    refused(INVALID, f, -1)
    refused(INVALID, f, 4, 1.0)
    refused(INVALID, f, 4, float("nan"))
    refused(INVALID, f, 4, 10000.0, "linear", 0.5)
    refused(INVALID, f, 4, 10000.0, "ntk", float("inf"))
    refused(INVALID, f, 4, 10000.0, "yarn", 2.0, 0.0)
    refused(INVALID, f, 4, 10000.0, "yarn", 2.0, 4096.0, 1.0, 1.0)
    refused(INVALID, f, 4, 10000.0, "yarn", 2.0, 4096.0, 32.0, 0.0)
    empty, _ = f(0)
    assert empty.numel() == 0


def test_table_bytes():
    assert binding.sparsp_rotary_table_bytes(binding.make_rotary((3, 0, 5), (10, 99, 7))) == (30 + 35) * 8
    # 2^31 entries and more are counted in 64 bits
    assert binding.sparsp_rotary_table_bytes(binding.make_rotary((64, 0, 0), (2 ** 30, 0, 0))) == 64 * 2 ** 33


def test_rotary_refused():
    shape = binding.make_shape(4, 64, (3, 4, 5), 2, 64)
    ok = binding.make_rotary((8, 8, 8), (3, 4, 5))
    p, ws = At(), At()

    def call(shape=shape, rotary=ok, table=p, positions=None, origin=(0, 0, 0), q=p, k=p, qo=p, ko=p, ws=ws):
        binding.sparsp_rotary_apply(shape, rotary, table, positions, origin, q, k, qo, ko, False, ws)

    changed = lambda s, **kw: type(s)(*[kw.get(n, getattr(s, n)) for n, _ in s._fields_])  # noqa: E731
    refused(INVALID, lambda: call(rotary=changed(ok, dtype=7)))
    refused(INVALID, lambda: call(rotary=changed(ok, pairing=2)))
    refused(INVALID, lambda: call(rotary=changed(ok, pairs_t=-1)))
    refused(INVALID, lambda: call(rotary=changed(ok, pairs_t=0, pairs_h=0, pairs_w=0)))
    refused(INVALID, lambda: call(rotary=changed(ok, len_h=0)))
    refused(UNSUPPORTED, lambda: call(rotary=changed(ok, rot_begin=-2)))
    refused(UNSUPPORTED, lambda: call(rotary=changed(ok, pairs_t=2 ** 30)))
    refused(INVALID, lambda: call(rotary=changed(ok, rot_begin=17)))  # 17 + 48 > 64
    refused(INVALID, lambda: call(rotary=changed(ok, len_h=3)))  # the grid has 4
    refused(INVALID, lambda: call(origin=(0, 0, 1)))
    refused(INVALID, lambda: call(origin=(-1, 0, 0)))
    refused(INVALID, lambda: call(origin=(2 ** 31 - 1, 0, 0)))
    refused(INVALID, lambda: call(shape=changed(shape, grid_w=0)))
    refused(UNSUPPORTED, lambda: call(shape=changed(shape, head_dim=60)))
    refused(UNSUPPORTED, lambda: call(shape=changed(shape, head_dim=264, stride_token=264)))
    refused(INVALID, lambda: call(shape=changed(shape, stride_token=60)))
    refused(INVALID, lambda: call(shape=changed(shape, stride_head=60)))
    refused(UNSUPPORTED, lambda: call(shape=changed(shape, grid_h=2 ** 20, grid_w=2 ** 20)))
    refused(UNSUPPORTED, lambda: call(shape=changed(shape, batch=2 ** 27)))
    refused(INVALID, lambda: call(q=None))
    refused(INVALID, lambda: call(q=At(4104)))
    refused(INVALID, lambda: call(ko=None))
    refused(INVALID, lambda: call(table=None))
    refused(INVALID, lambda: call(positions=At(4098)))
    refused(INVALID, lambda: call(positions=p, ws=None))
    refused(INVALID, lambda: call(ws=At(4100)))


def test_norm_refused():
    p = At()
    f = lambda **kw: binding.sparsp_layer_norm_fwd(binding.make_norm(**{"rows": 4, "dim": 64, **kw}), p, p, p, p, p, p)  # noqa: E731
    refused(INVALID, lambda: f(rows=-1))
    refused(INVALID, lambda: f(dim=0, stride_x=8, stride_y=8))
    refused(UNSUPPORTED, lambda: f(dim=16385))
    refused(INVALID, lambda: f(rows_per_group=-1))
    refused(INVALID, lambda: f(stride_x=63))
    refused(INVALID, lambda: f(stride_y=63))
    refused(INVALID, lambda: f(eps=-1.0))
    refused(INVALID, lambda: f(eps=float("nan")))
    refused(UNSUPPORTED, lambda: f(rows=2 ** 40, rows_per_group=1))
    norm = binding.make_norm(4, 64)
    bad = binding.make_norm(4, 64)
    bad.weight_dtype = binding.SPARSP_FP16
    refused(INVALID, lambda: binding.sparsp_layer_norm_fwd(bad, p, p, p, p, p, p))
    g = binding.sparsp_layer_norm_fwd
    refused(INVALID, g, norm, None, p, p, p, p, p)
    refused(INVALID, g, norm, p, p, p, None, p, p)
    refused(INVALID, g, norm, At(4097), p, p, p, p, p)
    refused(INVALID, g, norm, p, p, p, p, p, None)
    refused(INVALID, g, binding.make_norm(4, 64, stride_y=72), p, p, p, p, None, None)
    b, q = binding.sparsp_layer_norm_bwd, At(8192)
    refused(INVALID, b, norm, None, p, p, p, p, q, p, p, p)
    refused(INVALID, b, norm, p, q, p, None, p, p, p, p, p)
    refused(INVALID, b, norm, p, q, p, p, p, p, p, p, None)
    refused(INVALID, b, norm, p, q, p, p, p, p, p, p, At(4112))
    refused(INVALID, b, norm, p, q, p, p, p, q, p, p, p)  # dX = X
    refused(INVALID, b, binding.make_norm(4, 64, stride_y=72), p, q, p, p, p, p, p, p, p)
    assert binding.sparsp_layer_norm_workspace_bytes(norm) > 256


def test_ffn_refused():
    p = At()
    f = lambda **kw: binding.sparsp_gated_ffn_fwd(binding.make_ffn(**{"tokens": 4, "dim": 64, "hidden": 72, **kw}), p, p, p, p, p, p, p)  # noqa: E731
    refused(INVALID, lambda: f(tokens=-1))
    refused(UNSUPPORTED, lambda: f(tokens=2 ** 31))
    refused(UNSUPPORTED, lambda: f(dim=60))
    refused(UNSUPPORTED, lambda: f(hidden=76))
    refused(INVALID, lambda: f(hidden=0, stride_h=8))
    refused(INVALID, lambda: f(stride_x=56))
    refused(INVALID, lambda: f(stride_h=76))
    refused(INVALID, lambda: f(stride_w=68))
    ffn = binding.make_ffn(4, 64, 72)
    bad = binding.make_ffn(4, 64, 72)
    bad.dtype = binding.SPARSP_FP32
    refused(UNSUPPORTED, lambda: binding.sparsp_gated_ffn_fwd(bad, p, p, p, p, p, p, p))
    bad.dtype, bad.activation = 0, 3
    refused(INVALID, lambda: binding.sparsp_gated_ffn_fwd(bad, p, p, p, p, p, p, p))
    good = [p] * 7
    for i in (0, 1, 2, 3, 6):
        refused(INVALID, binding.sparsp_gated_ffn_fwd, ffn, *[None if i == j else a for j, a in enumerate(good)])
        refused(INVALID, binding.sparsp_gated_ffn_fwd, ffn, *[At(4104) if i == j else a for j, a in enumerate(good)])
    refused(INVALID, binding.sparsp_gated_ffn_fwd, ffn, p, p, p, p, p, None, p)
    good = [p] * 10
    for i in (0, 1, 2, 3, 4, 5, 8, 9):
        refused(INVALID, binding.sparsp_gated_ffn_bwd, ffn, *[None if i == j else a for j, a in enumerate(good)])
    assert binding.sparsp_gated_ffn_workspace_bytes(ffn, True) > binding.sparsp_gated_ffn_workspace_bytes(ffn, False)


@pytest.mark.parametrize("dim", [8, 5120, 18432, 18440])
@pytest.mark.parametrize("hidden", [8, 1000, 13824])
def test_a_workspace_for_more_tokens_serves_fewer(dim, hidden):
    need = [[binding.sparsp_gated_ffn_workspace_bytes(binding.make_ffn(m, dim, hidden), back) for back in (False, True)]
            for m in range(1, 600)]
    assert all(a[0] <= b[0] and a[1] <= b[1] for a, b in zip(need, need[1:]))
    assert all(forward <= backward for forward, backward in need)


@pytest.mark.parametrize("dim,pad,per", [(64, 0, 0), (1000, 1, 3), (1921, 0, 100), (5120, 4, 1), (12288, 0, 0)])
def test_a_norm_workspace_for_more_rows_serves_fewer(dim, pad, per):
    rows = sorted({*range(1, 70), *(int(1.1 ** k) for k in range(44, 140))})
    need = [binding.sparsp_layer_norm_workspace_bytes(binding.make_norm(r, dim, per, stride_x=dim + pad, stride_y=dim + pad))
            for r in rows]
    assert all(a <= b for a, b in zip(need, need[1:]))


@pytest.mark.parametrize("rows", [1, 5000])
def test_a_group_of_more_rows_than_there_can_be(rows):
    need = [binding.sparsp_layer_norm_workspace_bytes(binding.make_norm(rows, 64, per)) for per in (0, rows, 2 ** 62, 2 ** 63 - 1)]
    assert len(set(need)) == 1


def test_positions_as_tensors(monkeypatch):
    """They are passed by address: what would be misread there is refused here, and the stride is that of batch items."""
    seen = []

    class Library:
        def sparsp_rotary_apply(self, *args):
            seen.append(args[4])
            return binding.SPARSP_OK

    monkeypatch.setattr(binding, "lib", Library)
    shape, rotary, p = binding.make_shape(4, 64, (3, 4, 5), 2, 64, batch=2), binding.make_rotary((8, 8, 8), (3, 4, 5)), At()
    call = lambda pos: binding.sparsp_rotary_apply(shape, rotary, p, pos, (0, 0, 0), p, p, p, p, False, p)  # noqa: E731
    good = torch.zeros(2, 62, 3, dtype=torch.int32)
    padded = torch.zeros(2, 64, 3, dtype=torch.int32)[:, :62]
    for pos, stride in ((good, 62 * 3), (good[0], 0), (good[:1], 0), (good[:1].expand(2, -1, -1), 0), (padded, 64 * 3), (None, 0)):
        call(pos)
        assert seen.pop() == stride
    for bad in (good.long(), good.float(), good[:, :61], good[..., :2], good[0, 0], good[None], torch.cat((good, good)),
                torch.zeros(2, 3, 62, dtype=torch.int32).transpose(1, 2), torch.zeros(2, 62, 4, dtype=torch.int32)[..., :3],
                torch.zeros(62, 2, 3, dtype=torch.int32).transpose(0, 1)):
        with pytest.raises(ValueError):
            call(bad)
    assert not seen


def test_ffn_outputs_in_the_place_of_inputs():
    ffn = binding.make_ffn(4, 64, 64)
    x, wg, wu, h, gate, up, dh, dx, dwg, dwu, ws = (At(4096 * i) for i in range(1, 12))
    ok = [x, wg, wu, h, gate, up, ws]
    for out, into in ((3, 0), (3, 1), (4, 0), (5, 2), (4, 3), (5, 4)):
        args = list(ok)
        args[out] = ok[into]
        with pytest.raises(SparspError, match="output"):
            binding.sparsp_gated_ffn_fwd(ffn, *args)
    ok = [dh, x, wg, wu, gate, up, dx, dwg, dwu, ws]
    for out, into in ((6, 1), (7, 2), (8, 3), (6, 2), (8, 7)):
        args = list(ok)
        args[out] = ok[into]
        with pytest.raises(SparspError, match="output"):
            binding.sparsp_gated_ffn_bwd(ffn, *args)


@pytest.mark.parametrize("dim", [128, 1921, 5120])
@pytest.mark.parametrize("per", [1, 2, 16])
def test_a_norm_workspace_does_not_grow_with_small_groups(dim, per):
    """What a group of one worker's rows needs is nothing: 3.1 GB for 75600 x 5120 with a slot a group."""
    need = [binding.sparsp_layer_norm_workspace_bytes(binding.make_norm(r, dim, per)) for r in (75600, 10 ** 6)]
    assert need[0] == need[1] <= 128 << 20
