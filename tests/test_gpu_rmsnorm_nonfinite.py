"""Gains and outputs of fp4root_rmsnorm_quantize that are not finite: the group that holds one has
codes NaN and a scale that says so, the status is set, and the other groups are as ever."""
import math

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


def randn(shape, seed):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def none(codes):
    return (codes & 0x7F) == 0x7F


@pytest.mark.parametrize("e8m0", [False, True])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf, 3e38])
@pytest.mark.parametrize("rows,cols,at", [(5, 200, 40), (3, 96, 95), (2, 33, 32), (2, 3000, 2999), (1, 9000, 0)])
def test_gain(rows, cols, at, bad, e8m0):
    """3e38: finite, with outputs past the largest in some rows (the ones above 1.14 there)."""
    x = randn((rows, cols), rows + cols).bfloat16()
    x[:, at] = torch.where(torch.arange(rows, device="cuda") % 2 == 0, 8.0, 0.01).bfloat16()
    gain = 1 + 0.1 * randn((cols,), 3)
    plain = {g: F.fp4root_rmsnorm_quantize(x, gain, group=g, e8m0=e8m0) for g in (0, 32, 64, 128)}
    gain[at] = bad
    for g in (0, 32, 64, 128):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        o = F.fp4root_rmsnorm_quantize(x, gain, group=g, e8m0=e8m0, status=status, want_y=True)
        assert int(status) == -4
        k = at // g if g else 0
        lo, hi = (k * g, min(k * g + g, cols)) if g else (0, cols)
        y = (x.float() * o.rstd[:, None] * gain)[:, lo:hi]
        wrong = ~torch.isfinite(y).all(1)
        assert bool(wrong[0]) and bool(wrong.all()) == (not math.isfinite(bad) or rows == 1)
        scales = o.scales.view(rows, -1)
        assert bool(none(o.codes[wrong, lo:hi]).all())
        if e8m0:
            assert bool((scales[wrong, k] == 255).all())
        else:
            assert not bool(torch.isfinite(scales[wrong, k]).any())
            assert torch.equal(torch.isnan(scales[wrong, k]), torch.isnan(y[wrong]).any(1))
        assert not bool(none(o.codes[~wrong]).any())
        rest = [c for c in range(cols) if not lo <= c < hi]
        assert torch.equal(o.codes[:, rest], plain[g].codes[:, rest])
        others = [j for j in range(scales.shape[1]) if j != k]
        assert torch.equal(scales[:, others], plain[g].scales.view(rows, -1)[:, others])
        assert torch.equal(o.rstd, plain[g].rstd)


@pytest.mark.parametrize("e8m0", [False, True])
@pytest.mark.parametrize("group", [0, 32, 128])
def test_row_of_the_stream(group, e8m0):
    """A NaN or an infinity in the stream reaches every group of its row, its scales too."""
    for bad in (math.nan, math.inf):
        x = randn((6, 300), 9).bfloat16()
        clean = F.fp4root_rmsnorm_quantize(x, group=group, e8m0=e8m0)
        x[4, 150] = bad
        o = F.fp4root_rmsnorm_quantize(x, group=group, e8m0=e8m0)
        assert bool(none(o.codes[4]).all()) and math.isnan(float(o.rstd[4]))
        s = o.scales.view(6, -1)
        assert bool((s[4] == 255).all()) if e8m0 else bool(torch.isnan(s[4]).all())
        rows = [0, 1, 2, 3, 5]
        assert torch.equal(o.codes[rows], clean.codes[rows]) and torch.equal(s[rows], clean.scales.view(6, -1)[rows])
