"""A list that says more CTAs than the workspace and the table have places for is none that a table was made for."""
import pytest

from paper_2609_32197_b200 import binding
from test_layer_host import At, INVALID, no_stream, refused  # noqa: F401
from test_step_host import grads, table_of


@pytest.mark.parametrize("change", [{"ctas": 8 * 148 + 1}, {"ctas": 1 << 20}, {"ctas": 0}, {"ctas": -1}, {"chunks": -1}])
def test_refused(change):
    lst = grads((4096, 8), (8192, 8))
    binding.sparsp_grad_table(lst, table_of(lst))
    lst.table = At(1 << 16)
    for k, v in change.items():
        setattr(lst, k, v)
    refused(INVALID, binding.sparsp_grad_squares, lst, At(1 << 20))
    refused(INVALID, binding.sparsp_grad_clip, lst, 1.0, None, At(1 << 20))


def test_the_most_that_there_are():
    lst = grads((1 << 20, 1 << 30))
    binding.sparsp_grad_table(lst, table_of(lst))
    assert lst.ctas == 8 * 148 and 512 + lst.ctas * 8 <= binding.sparsp_grad_workspace_bytes()
