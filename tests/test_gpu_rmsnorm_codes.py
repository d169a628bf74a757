"""FP32 scales and E4M3 codes of fp4root_rmsnorm_quantize, bit for bit.

With the device's own h and rstd, y = fl32(fl32(h rstd) gain) has one value, and so have amax,
s = fl32(amax / 448), the inverse fl32(448 / amax) and the code E4M3(fl32(y inverse)): nothing here
has a tolerance.  Both quotients are taken in binary64 and rounded from there, which is the rounding
of the exact quotient: amax has 24 bits and 448 = 7 2^6, so amax / 448 lies at least 2^-28
(relative) from every binary32 midpoint, and 448 / amax at least 2^-49, while binary64 is off by
2^-53.  Ratios of 16-bit values in a row fall on ties of E4M3 by themselves, so an inverse that is
one place off shows in some codes of every few rows."""

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


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def check_fp32_scales(x, residual, gain, group, **kw):
    o = F.fp4root_rmsnorm_quantize(x, gain, residual, group=group, **kw)
    rows, cols = x.shape
    y = o.h.float() * o.rstd[:, None]
    if gain is not None:
        y = y * gain.float()
    y = y.cpu()
    g = group or cols
    groups = -(-cols // g)
    full = torch.nn.functional.pad(y, (0, groups * g - cols)).view(rows, groups, g)
    amax = full.abs().amax(2).clamp_min(2.0 ** -100).double()
    assert torch.equal(o.scales.cpu().view(rows, groups), (amax / 448.0).float())
    inverse = (448.0 / amax).float()
    want = (full * inverse[:, :, None]).to(torch.float8_e4m3fn).view(torch.uint8).view(rows, -1)[:, :cols]
    assert torch.equal(o.codes.cpu(), want)
    return o


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,cols,group", [(64, 8192, 0), (37, 5003, 128), (300, 96, 32), (65, 1001, 64), (3, 20000, 0)])
def test_codes_and_scales(rows, cols, group, dtype):
    g = gen(rows + cols)
    x = (torch.randn(rows, cols, generator=g, device="cuda") * 3).to(dtype)
    r = (torch.randn(rows, cols, generator=g, device="cuda") * 4).to(dtype)
    gain = (1 + 0.1 * torch.randn(cols, generator=g, device="cuda")).bfloat16()
    check_fp32_scales(x, r, gain, group)
    check_fp32_scales(x, None, gain.float(), group)
    check_fp32_scales(x, None, None, group)
