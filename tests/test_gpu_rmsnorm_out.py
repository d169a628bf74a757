"""Results of fp4root_rmsnorm_quantize that are given to a later call as `out`."""
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


def randn(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


@pytest.mark.parametrize("strided", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_call_without_residual_lends_no_output(dtype, strided):
    """The first norm of a model has no residual, the next ones have: the first stream stays."""
    cut = (lambda t: t[:, 3:99]) if strided else (lambda t: t[:, :96].contiguous())
    x, x2, r = (cut(randn((7, 100), dtype, k)) for k in range(3))
    keep, keep2 = x.clone(), x2.clone()
    o = F.fp4root_rmsnorm_quantize(x, group=32, want_y=True)
    assert o.h is x
    first = [t.clone() for t in o]
    want = F.fp4root_rmsnorm_quantize(x2, None, r, group=32, want_y=True)
    alone = F.fp4root_rmsnorm_quantize(x2, group=32, want_y=True)
    got = F.fp4root_rmsnorm_quantize(x2, None, r, group=32, out=o)
    assert torch.equal(x, keep) and torch.equal(x2, keep2) and got.h is not x and got.h is not x2
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert got.codes is o.codes and got.scales is o.scales and got.rstd is o.rstd and got.y is o.y
    # one with a residual keeps its h, and lends it to no call without one
    again = F.fp4root_rmsnorm_quantize(x2, None, r, group=32, out=got)
    assert again.h is got.h
    plain = F.fp4root_rmsnorm_quantize(x, group=32, out=again)
    assert plain.h is x and torch.equal(again.h, want.h) and all(torch.equal(a, b) for a, b in zip(plain, first))
    # ... whose result lends no stream either, also where a field but h is replaced
    for lent in (plain, plain._replace(y=torch.empty_like(plain.y)),
                 F.fp4root_rmsnorm_quantize(x2, group=32, out=plain)):
        assert torch.equal(F.fp4root_rmsnorm_quantize(x2, None, r, group=32, out=lent).h, want.h)
        assert torch.equal(x, keep) and torch.equal(x2, keep2)
    assert all(torch.equal(a, b) for a, b in zip(F.fp4root_rmsnorm_quantize(x2, group=32, out=plain), alone))


def test_in_place_where_the_caller_says_so():
    """h=x, or the residual, by _replace: written, as the caller asks."""
    x, r = randn((5, 64), torch.bfloat16, 4), randn((5, 64), torch.bfloat16, 5)
    want = F.fp4root_rmsnorm_quantize(x, None, r).h
    o = F.fp4root_rmsnorm_quantize(x)
    a, b = x.clone(), r.clone()
    got = F.fp4root_rmsnorm_quantize(a, None, r, out=o._replace(h=a))
    assert got.h is a and torch.equal(a, want)
    got = F.fp4root_rmsnorm_quantize(x, None, b, out=o._replace(h=b))
    assert got.h is b and torch.equal(b, want)
    assert F.fp4root_rmsnorm_quantize(x, None, r, out=o._replace(h=None)).h is None      # not wanted
