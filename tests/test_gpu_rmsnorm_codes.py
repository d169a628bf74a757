"""FP32 scales and E4M3 codes of fp4root_rmsnorm_quantize, bit for bit.

With the device's own h and rstd, y = fl32(fl32(h rstd) gain) has one value, and so have amax,
s = fl32(amax / 448), the inverse fl32(448 / amax) and the code E4M3(fl32(y inverse)): nothing here
has a tolerance.  Both quotients are taken in binary64 and rounded from there, which is the rounding
of the exact quotient: amax has 24 bits and 448 = 7 2^6, so amax / 448 lies at least 2^-28
(relative) from every binary32 midpoint, and 448 / amax at least 2^-49, while binary64 is off by
2^-53.  Ratios of 16-bit values in a row fall on ties of E4M3 by themselves, so an inverse that is
one place off shows in some codes of every few rows."""
import ctypes

import pytest
import torch

from paper_2607_04422_amd import build
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
@pytest.mark.parametrize("rows,cols,group", [(64, 8192, 0), (37, 5003, 128), (300, 96, 32), (65, 1001, 64),
                                             (3, 20000, 0)])
def test_codes_and_scales(rows, cols, group, dtype):
    g = gen(rows + cols)
    x = (torch.randn(rows, cols, generator=g, device="cuda") * 3).to(dtype)
    r = (torch.randn(rows, cols, generator=g, device="cuda") * 4).to(dtype)
    gain = (1 + 0.1 * torch.randn(cols, generator=g, device="cuda")).bfloat16()
    check_fp32_scales(x, r, gain, group)
    check_fp32_scales(x, None, gain.float(), group)
    check_fp32_scales(x, None, None, group)


@pytest.mark.parametrize("group", [0, 32])
@pytest.mark.parametrize("top", [1e19, 2e19, 8e37, 9e37, 1.2e38, 2e38, 3.4e38])
def test_large_finite_outputs(top, group):
    """A group's largest output up to the largest binary32 value: 448 / amax is about 1e-36 there,
    an ordinary number, though 1 / amax is subnormal."""
    x = torch.randn(5, 96, generator=gen(7), device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    unit = F.fp4root_rmsnorm_quantize(x, None, group=group, quantize=False, want_y=True).y
    gain = torch.full((96,), top / float(unit.abs().max()) * (1 - 2.0 ** -20), device="cuda")
    gain[:32] *= 2.0 ** -90                          # an ordinary group beside it
    o = check_fp32_scales(x, None, gain, group, status=status, want_y=True)
    assert bool(torch.isfinite(o.y).all()) and int(status) == 0
    assert torch.equal(o.y, unit * gain) and float(o.y.abs().max()) > top / 4
    codes = o.codes.view(torch.float8_e4m3fn).float().abs()
    assert float(codes.max()) == 448.0
    e = F.fp4root_rmsnorm_quantize(x, gain, group=group, e8m0=True, status=status)
    assert float(e.codes.view(torch.float8_e4m3fn).float().abs().max()) > 220 and int(status) == 0


def test_quotients_by_448_every_value():
    """Every amax in [2^-100, FLT_MAX] against binary64 divisions on the device."""
    lib = ctypes.CDLL(build.SWEEPS)
    out = torch.zeros(2, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    first = 0x0D800000
    count = 0x7F7FFFFF - first + 1
    u, where = ctypes.c_uint32, ctypes.c_void_p(out.data_ptr())
    assert lib.fp4root_sweep_448(u(first), u(count), where, None) == 0
    torch.cuda.synchronize()
    bad, which = (int(v) & 0xFFFFFFFF for v in out)
    assert bad == 0, f"{bad} differ, one of them {which:#010x}"
