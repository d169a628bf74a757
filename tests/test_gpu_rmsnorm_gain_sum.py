"""The join of the gain gradient's partial rows (fp4root_rmsnorm_backward)."""
import pytest
import torch

from tests.gpu_util import need_gpu

pytestmark = pytest.mark.gpu

F = None


def setup_module():
    global F
    need_gpu()
    from paper_2607_04422_amd import fp4root
    F = fp4root


@pytest.mark.parametrize("rows,cols", [(200, 4096), (256, 4001), (255, 12000), (3, 2500), (131, 5003)])
def test_cancelling_workgroups(rows, cols):
    """At these widths a row is a workgroup and there are no more rows than workgroups, so that a
    partial is one product, exact here: h = rstd = 1 makes dgain the sum of dy.  Two rows of
    opposite sign cancel, and what is left is exact in binary32; added there one after the other,
    2^25 + 1 would lose the 1."""
    h, rstd = torch.ones(rows, cols, device="cuda"), torch.ones(rows, device="cuda")
    dy = torch.ones(rows, cols, device="cuda")
    col = torch.arange(cols, device="cuda")
    first = col % (rows - 1)
    last = first + 1 + (col // 7) % (rows - 1 - first)          # first < last < rows
    size = 2.0 ** (25 + col % 28).float()                        # at most 2^52: exact in binary64 beside ones
    dy[first, col], dy[last, col] = size, -size
    _, dgain = F.fp4root_rmsnorm_backward(dy, h, None, rstd)
    assert torch.equal(dgain, torch.full_like(dgain, rows - 2.0))
