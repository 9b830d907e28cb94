"""Widths at which rows are shared out in other ways than at the widths of test_gpu_gated_norm.py, by that file's test."""
import pytest

from test_gpu_gated_norm import BF, FL, HF
from test_gpu_gated_norm import test_forward_and_backward as whole

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("norm_y,norm_r", [("none", "layer"), ("layer", "layer"), ("rms", "none")])
@pytest.mark.parametrize("rows,dim,groups,dtype,wtype", [
    (700, 2568, 1, BF, FL), (1000, 2816, 3, BF, BF), (601, 3328, 1, HF, FL), (450, 3456, 1, BF, BF), (900, 3584, 5, BF, FL),
    (299, 3840, 1, HF, HF), (600, 4096, 300, BF, FL), (297, 4608, 1, BF, BF), (301, 5128, 1, BF, FL), (4, 7736, 1, BF, FL),
    (301, 8192, 2, BF, FL), (150, 8192, 1, FL, FL), (3000, 256, 1, BF, FL), (2500, 392, 6, HF, HF), (1500, 256, 1, FL, FL)])
def test_widths(rows, dim, groups, dtype, wtype, norm_y, norm_r):
    whole(rows, dim, groups, dtype, wtype, norm_y, norm_r)
