"""Groups of more rows than there are, up to the largest number that a description holds, are one group of all rows."""
import pytest
import torch

from paper_2609_32197_b200 import binding
from test_gpu_gated_norm import BF, EPS, FL, backward, forward, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,dim", [(1, 64), (2, 1032), (3, 64), (500, 520)])
@pytest.mark.parametrize("more", [1, 1 << 40, (1 << 62) + 1, (1 << 63) - 1])
def test_groups_of_more_rows_than_there_are(rows, dim, more):
    v = inputs(rows, dim, 1, BF, FL, 3)
    out = []
    for per in (0, rows if more == 1 else more, rows + 1):
        step = binding.make_gated_norm(rows, dim, per, "rms", "layer", EPS, BF, FL)
        got = forward(step, v, "rms", "layer")
        ws = binding.make_gated_norm_workspace(step)
        ws[256:].fill_(255)
        out.append({**got, **backward(step, v, got["r"], got["stats_y"], got["stats_r"], ws)})
    for other in out[1:]:
        for k, t in out[0].items():
            assert not bool(t.isnan().any()) and torch.equal(other[k], t), k
