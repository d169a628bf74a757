"""RMS norm and its gradients at sizes where the kernels take further turns: more wide rows than
workgroups, chunks of more than 64 rows for the gain's gradient, and inputs past the size up to
which they are read through the caches."""
import pytest
import torch

from tests.gpu_util import need_gpu

pytestmark = pytest.mark.gpu

F = None
U = 2.0 ** -24


def setup_module():
    global F
    need_gpu()
    from paper_2607_04422_amd import fp4root
    F = fp4root


def randn(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").mul_(scale).to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,cols", [(600, 16400), (600, 32768), (4500, 16400), (1030, 24577), (520, 32765)])
def test_gradients_of_many_wide_rows(rows, cols, dtype):
    """dx as in test_gpu_rmsnorm.check_backward: 8 roundings on any term, 64 in the mean, one to the
    type.  dgain: a wave adds up to 20 rows (chunks of 64 to 73 rows, four waves, four rows a turn),
    each term rounded once more in its product, then four waves; the join is binary64, and one
    rounding: fewer than 32 2^-24 of the magnitudes' sum."""
    h, dy, dh = (randn((rows, cols), dtype, rows + cols + k, s) for k, s in enumerate((3.0, 0.1, 0.1)))
    gain = randn((cols,), torch.float32, 5)
    h[rows // 2] = 0.0
    rstd = F.fp4root_rmsnorm_quantize(h, gain, eps=1e-3, quantize=False).rstd
    dx, dgain = F.fp4root_rmsnorm_backward(dy, h, gain, rstd, dh=dh)
    over = dy.clone()
    F.fp4root_rmsnorm_backward(over, h, gain, rstd, dh=dh, dx=over, want_dgain=False)
    assert torch.equal(over, dx)
    half, tiny = {torch.float32: (U, 2.0 ** -149), torch.bfloat16: (2.0 ** -8, 2.0 ** -133),
                  torch.float16: (2.0 ** -11, 2.0 ** -24)}[dtype]
    want_g = torch.zeros(cols, dtype=torch.float64, device="cuda")
    size_g = torch.zeros_like(want_g)
    for a in range(0, rows, 256):                     # the formula, 256 rows at a time
        at = slice(a, a + 256)
        r, d = rstd[at].double()[:, None], dy[at].double()
        xh, g, e = h[at].double() * r, d * gain.double(), dh[at].double()
        mean, size = (g * xh).mean(1, keepdim=True), (g * xh).abs().mean(1, keepdim=True)
        want = r * (g - xh * mean) + e
        tol = 8 * U * (r * g.abs() + r * (xh * mean).abs() + e.abs()) + 64 * U * r * xh.abs() * size
        assert bool(((dx[at].double() - want).abs() <= tol + half * (want.abs() + tol) + tiny).all()), a
        want_g += (d * xh).sum(0)
        size_g += (d * xh).abs().sum(0)
    assert bool(((dgain.double() - want_g).abs() <= 32 * U * size_g).all())
    if rows <= 600:
        return
    # the last rows alone: the same bits
    part = slice(rows - 3, rows)
    alone = F.fp4root_rmsnorm_backward(dy[part], h[part], gain, rstd[part], dh=dh[part], want_dgain=False)[0]
    assert torch.equal(alone, dx[part])


@pytest.mark.parametrize("rows,cols,dtype,residual", [
    (8200, 8201, torch.bfloat16, True), (4100, 8200, torch.float32, True), (1100, 32768, torch.float32, False),
    (600, 32768, torch.bfloat16, True), (530000, 128, torch.float16, True)])
def test_forward_past_the_caches(rows, cols, dtype, residual):
    """Inputs of more than 128 MiB (and one of 600 wide rows): scales and codes bit for bit, and the
    same bits as a few of the rows give alone."""
    x, gain = randn((rows, cols), dtype, rows, 3.0), randn((cols,), torch.bfloat16, 6)
    r = randn((rows, cols), dtype, cols, 2.0) if residual else None
    o = F.fp4root_rmsnorm_quantize(x, gain, r, eps=1e-5)
    mx = F.fp4root_rmsnorm_quantize(x, gain, r, eps=1e-5, group=32, e8m0=True)
    assert torch.equal(mx.rstd, o.rstd) and torch.equal(mx.h, o.h)
    step = (1 << 25) // cols                          # rows at a time
    for a in range(0, rows, step):
        at = slice(a, a + step)
        h = x[at] if r is None else (x[at].float() + r[at].float()).to(dtype)
        assert torch.equal(o.h[at], h)
        want = (h.double().square().mean(1) + 1e-5).rsqrt()
        assert bool(((o.rstd[at].double() - want).abs() <= (U + 2.0 ** -40) * want).all())
        y = h.float() * o.rstd[at][:, None] * gain.float()
        amax = y.abs().amax(1).double()
        assert torch.equal(o.scales[at], torch.div(amax, torch.full_like(amax, 448.0)).float())
        inverse = torch.div(torch.full_like(amax, 448.0), amax).float()
        codes = (y * inverse[:, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        assert torch.equal(o.codes[at], codes)
    for part in (slice(0, 5), slice(rows - 5, rows)):
        rp = None if r is None else r[part]
        alone = F.fp4root_rmsnorm_quantize(x[part], gain, rp, eps=1e-5, group=32, e8m0=True)
        assert torch.equal(alone.codes, mx.codes[part]) and torch.equal(alone.scales, mx.scales[part])
        assert torch.equal(alone.rstd, mx.rstd[part])
