"""Root-mean-square norm with the residual's addition and its 8-bit output
(fp4root_rmsnorm_quantize), and its gradients (fp4root_rmsnorm_backward).

Tolerances.  h is compared bit for bit.  rstd is a binary64 value rounded once: 2^-24 (and
2^-40 for the sum and the root).  With the device's own h and rstd, y = fl32(fl32(h rstd) gain)
has one value, so amax, E8M0 scales and the codes under them are compared bit for bit; an FP32
scale is within half a step, 2^-24, of amax / 448 (and 2^-50 for the quotient's rounding in
binary64), and a code under it within half a step of E4M3 of y 448 / amax, where the inverse
scale and its product round once each (2 2^-24).  Gradients: see `check_backward`."""
import math

import numpy as np
import pytest
import torch

from tests.gpu_util import need_gpu

pytestmark = pytest.mark.gpu

F = None
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def setup_module():
    global F
    need_gpu()
    from paper_2607_04422_amd import fp4root
    F = fp4root


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(shape, dtype, seed, scale=1.0):
    return (torch.randn(shape, generator=gen(seed), device="cuda") * scale).to(dtype)


def np64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def e4m3_step(v):
    """E4M3's spacing at magnitude v."""
    e = np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -6)))
    return 2.0 ** (e - 3)


def check_forward(x, res, gain, o, group, e8m0, eps):
    dtype = x.dtype
    h = x if res is None else (x.float() + res.float()).to(dtype)
    assert torch.equal(o.h, h)
    cols = x.shape[-1]
    h64 = np64(h).reshape(-1, cols)
    rstd = np64(o.rstd).reshape(-1, 1)
    want = 1.0 / np.sqrt((h64 * h64).sum(1, keepdims=True) / cols + eps)
    # one below 2^-126 is a multiple of 2^-149, off by half of that at most
    assert np.all(np.abs(rstd - want) <= (2.0 ** -24 + 2.0 ** -40) * want + 2.0 ** -150)
    y = h.float().reshape(-1, cols) * o.rstd.reshape(-1, 1)
    if gain is not None:
        y = y * gain.float()
    if o.y is not None:
        assert torch.equal(o.y.reshape(-1, cols), y.to(dtype))
    if o.codes is None:
        return
    y = y.cpu().numpy()
    g = group or cols
    codes = o.codes.reshape(-1, cols).cpu().view(torch.float8_e4m3fn).float().numpy().astype(np.float64)
    scales = o.scales.reshape(y.shape[0], -1).cpu()
    assert scales.shape[1] == -(-cols // g)
    for k in range(scales.shape[1]):
        part = y[:, k * g:(k + 1) * g]
        got = codes[:, k * g:(k + 1) * g]
        amax = np.maximum(np.abs(part).max(1), np.float32(2.0 ** -100)).astype(np.float64)
        if e8m0:
            e = scales[:, k].numpy().astype(np.int64) - 127
            fits = amax <= 448.0 * 2.0 ** e
            assert fits.all() and not (amax <= 448.0 * 2.0 ** (e - 1)).any()
            exact = torch.from_numpy((part.astype(np.float64) * 2.0 ** -e[:, None]).astype(np.float32))
            assert np.array_equal(got, exact.to(torch.float8_e4m3fn).float().numpy().astype(np.float64))
        else:
            s = scales[:, k].numpy().astype(np.float64)
            assert np.all(np.abs(s - amax / 448.0) <= (2.0 ** -24 + 2.0 ** -50) * amax / 448.0)
            v = part.astype(np.float64) * (448.0 / amax)[:, None]
            assert np.all(np.abs(got - v) <= e4m3_step(v) / 2 + 2 * 2.0 ** -24 * np.abs(v))


SHAPES = [(1, 1), (1, 4096), (3, 7), (5, 8), (2, 31), (4, 33), (7, 512), (3, 513), (2, 1024), (5, 1025), (9, 2048),
          (1, 2049), (3, 4096), (2, 5003), (2, 8192), (3, 8200), (1, 16384), (2, 16391), (1, 32768), (513, 96),
          (130, 1000), (33, 129), (35, 256), (17, 257), (6, 1536), (3, 2560), (2, 6145), (520, 8193), (700, 2057),
          (150, 16400)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_forward(rows, cols, dtype):
    x = randn((rows, cols), dtype, rows * 7 + cols, 3.0)
    res = randn((rows, cols), dtype, rows + cols, 2.0)
    k = 0
    for group in (0, 32, 64, 128):
        for e8m0 in (False, True):
            k += 1
            gain = None if k % 4 == 0 else randn((cols,), (torch.float32, torch.bfloat16)[k % 2], 5 + k)
            r = res if k % 3 else None
            o = F.fp4root_rmsnorm_quantize(x, gain, r, eps=1e-5, group=group, e8m0=e8m0, want_y=k % 2 == 0)
            check_forward(x, r, gain, o, group, e8m0, 1e-5)


@pytest.mark.parametrize("dtype", TYPES)
def test_forward_without_codes(dtype):
    x, res = randn((6, 300), dtype, 1), randn((6, 300), dtype, 2)
    gain = randn((300,), torch.bfloat16, 3)
    o = F.fp4root_rmsnorm_quantize(x, gain, res, quantize=False, want_y=True)
    assert o.codes is None and o.scales is None
    check_forward(x, res, gain, o, 0, False, 1e-6)


@pytest.mark.parametrize("group,e8m0", [(0, False), (0, True), (32, False), (128, True)])
def test_zero_rows_and_tiny_and_huge_values(group, e8m0):
    """Padding rows, a row of subnormals, the type's largest values, one hot column."""
    x = randn((8, 160), torch.float32, 4)
    x[1] = 0.0
    x[2] = 1e-41
    x[3] = 3e38
    x[4, :] = 0.0
    x[4, 77] = 1e30
    x[5, 32:64] = 0.0
    gain = torch.ones(160, device="cuda")
    gain[5] = 0.0
    o = F.fp4root_rmsnorm_quantize(x, gain, eps=1e-30, group=group, e8m0=e8m0)
    check_forward(x, None, gain, o, group, e8m0, 1e-30)
    assert int((o.codes[1] & 0x7F).max()) == 0 and bool(torch.isfinite(o.rstd).all())
    # a scale is never 0, so that a reader may divide by it
    assert float(o.scales.float().min()) > 0


def test_non_finite_rows_stay_alone():
    for bad in (math.nan, math.inf, -math.inf):
        x = randn((6, 200), torch.bfloat16, 5)
        clean = F.fp4root_rmsnorm_quantize(x, group=32)
        x[3, 150] = bad
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        o = F.fp4root_rmsnorm_quantize(x, group=32, status=status)
        assert int(status) == -4
        assert math.isnan(float(o.rstd[3]))
        assert bool(((o.codes[3] & 0x7F) == 0x7F).all())
        rows = [0, 1, 2, 4, 5]
        assert torch.equal(o.codes[rows], clean.codes[rows]) and torch.equal(o.scales[rows], clean.scales[rows])
        assert torch.equal(o.rstd[rows], clean.rstd[rows])
    status = torch.full((1,), 9, dtype=torch.int32, device="cuda")
    x[3, 150] = 0.0
    F.fp4root_rmsnorm_quantize(x, status=status)
    assert int(status) == 9                                   # left as it was
    # float16: a sum past the largest is an infinity of the stream
    big = torch.full((2, 64), 6e4, dtype=torch.float16, device="cuda")
    F.fp4root_rmsnorm_quantize(big, residual=big, status=status)
    assert int(status) == -4
    # an infinite gain: its group's codes are not numbers, the others' are
    gain = torch.ones(200, device="cuda")
    gain[40] = math.inf
    for e8m0 in (False, True):
        status.zero_()
        o = F.fp4root_rmsnorm_quantize(x, gain, group=32, e8m0=e8m0, status=status)
        assert int(status) == -4
        assert bool(((o.codes[:, 40] & 0x7F) == 0x7F).all())
        plain = F.fp4root_rmsnorm_quantize(x, None, group=32, e8m0=e8m0)
        assert torch.equal(o.codes[:, 64:], plain.codes[:, 64:])
        # a gain that is no number: its own codes are none either
        nan = torch.where(torch.isinf(gain), math.nan, gain)
        o = F.fp4root_rmsnorm_quantize(x, nan, group=32, e8m0=e8m0)
        assert bool(((o.codes[:, 40] & 0x7F) == 0x7F).all())
        assert torch.equal(o.codes[:, 64:], plain.codes[:, 64:])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [96, 515, 4099])
def test_strides_in_place_and_untouched(dtype, cols):
    """Rows of one stride inside wider buffers at odd offsets, h over the residual or over x, and
    what lies between the rows left alone."""
    wide = randn((11, cols + 13), dtype, 6, 2.0)
    x = wide[:, 3:3 + cols]
    other = randn((11, 2 * cols + 1), dtype, 7)
    res = other[:, cols:2 * cols]
    gain = randn((cols,), torch.float32, 8)
    want = F.fp4root_rmsnorm_quantize(x.contiguous(), gain, res.contiguous(), group=32, want_y=True)
    check_forward(x.contiguous(), res.contiguous(), gain, want, 32, False, 1e-6)
    got = F.fp4root_rmsnorm_quantize(x, gain, res, group=32, want_y=True)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    keep, before = other.clone(), wide.clone()
    out = got._replace(h=res, y=x)               # over both inputs
    F.fp4root_rmsnorm_quantize(x, gain, res, group=32, out=out)
    assert torch.equal(res, want.h) and torch.equal(x, want.y)
    assert torch.equal(out.codes, want.codes) and torch.equal(out.scales, want.scales)
    keep[:, cols:2 * cols] = want.h
    before[:, 3:3 + cols] = want.y
    assert torch.equal(other, keep) and torch.equal(wide, before)
    with pytest.raises(F.Fp4RootError):          # half over the residual
        F.fp4root_rmsnorm_quantize(res, gain, res, group=32, out=got._replace(h=other[:, cols - 1:2 * cols - 1]))
    with pytest.raises(ValueError):
        F.fp4root_rmsnorm_quantize(wide.t(), None)
    with pytest.raises(ValueError):
        F.fp4root_rmsnorm_quantize(x, gain, group=64, out=got)
    with pytest.raises(TypeError):
        F.fp4root_rmsnorm_quantize(x, gain.half())


def test_leading_dimensions_and_empty():
    x = randn((2, 3, 5, 64), torch.bfloat16, 9)
    o = F.fp4root_rmsnorm_quantize(x, group=32)
    assert o.codes.shape == x.shape and o.scales.shape == (2, 3, 5, 2) and o.rstd.shape == (2, 3, 5)
    check_forward(x, None, None, o, 32, False, 1e-6)
    with pytest.raises(ValueError):              # columns 64 apart
        F.fp4root_rmsnorm_quantize(x[:, :, :, 0])
    e = F.fp4root_rmsnorm_quantize(x[:0], residual=x[:0])
    assert e.codes.shape == (0, 3, 5, 64)
    dx, dg = F.fp4root_rmsnorm_backward(x[:0], x[:0], None, torch.empty((0, 3, 5), device="cuda"))
    assert dx.shape == (0, 3, 5, 64) and float(dg.abs().max()) == 0.0
    v = x[0, 0, 0]
    check_forward(v, None, None, F.fp4root_rmsnorm_quantize(v), 0, False, 1e-6)


def test_far_rows():
    """Rows past 2^32 elements from the first, and more rows than one launch takes."""
    buf = torch.zeros((1 << 32) + 4096, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((3, 128), ((1 << 31) + 8, 1))
    x.copy_(randn((3, 128), torch.bfloat16, 10))
    o = F.fp4root_rmsnorm_quantize(x, group=64)
    check_forward(x.contiguous(), None, None, o._replace(h=o.h.contiguous()), 64, False, 1e-6)
    rows = (1 << 21) + 3
    x = buf[:rows * 8].view(rows, 8).normal_(generator=gen(11))
    o = F.fp4root_rmsnorm_quantize(x)
    part = slice(rows - 5, rows)
    check_forward(x[part], None, None, F.RmsNormOutput(o.codes[part], o.scales[part], o.rstd[part], x[part], None), 0,
                  False, 1e-6)
    dx, dg = F.fp4root_rmsnorm_backward(x, x, None, o.rstd)
    check_backward(x[part], x[part], None, o.rstd[part], None, dx[part], None, 1e-6)
    xh = x.double() * o.rstd.double()[:, None]
    want, size = (x.double() * xh).sum(0), (x.double() * xh).abs().sum(0)
    assert bool(((dg.double() - want).abs() <= (rows / 256 + 64) * 2.0 ** -24 * size).all())


def check_backward(dy, h, gain, rstd, dh, dx, dgain, eps):
    """Against the formula in binary64.  dx = rstd (g - xhat mean) + dh in binary32 from rounded
    factors: at most 8 roundings on any term, so 8 2^-24 of the terms' magnitudes; the mean adds
    at most 32 products in a thread, 6 steps over a wave and 16 waves, each of which rounds by
    2^-24 of the sum of magnitudes at most: 64 2^-24 of it; then one rounding to the type.  dgain
    adds up to 16 rows or rows / 256 in a thread, 32 slots, up to 8 partials and then 64 slices in 6
    steps: each addition rounds by 2^-24 of the magnitudes' sum at most, fewer than rows / 256 + 64
    of them one after another."""
    cols = h.shape[-1]
    d, x, r = np64(dy).reshape(-1, cols), np64(h).reshape(-1, cols), np64(rstd).reshape(-1, 1)
    g = d if gain is None else d * np64(gain)
    xh = x * r
    mean = (g * xh).mean(1, keepdims=True)
    e = np.zeros_like(x) if dh is None else np64(dh).reshape(-1, cols)
    want = r * (g - xh * mean) + e
    u = 2.0 ** -24
    tol = 8 * u * (r * np.abs(g) + r * np.abs(xh * mean) + np.abs(e)) + 64 * u * r * np.abs(xh) * np.abs(g * xh).mean(1, keepdims=True)
    half, tiny = {torch.float32: (u, 2.0 ** -149), torch.bfloat16: (2.0 ** -8, 2.0 ** -133),
                  torch.float16: (2.0 ** -11, 2.0 ** -24)}[h.dtype]
    got = np64(dx).reshape(-1, cols)
    bad = np.abs(got - want) > tol + half * (np.abs(want) + tol) + tiny
    assert not bad.any(), (int(bad.sum()), np.abs(got - want).max())
    if dgain is not None:
        k = x.shape[0] / 256 + 64
        assert np.all(np.abs(np64(dgain) - (d * xh).sum(0)) <= k * u * np.abs(d * xh).sum(0))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES + [(1025, 64), (4099, 200)])
def test_backward(rows, cols, dtype):
    h = randn((rows, cols), dtype, rows * 3 + cols, 3.0)
    h[rows // 2] = 0.0
    dy = randn((rows, cols), dtype, rows + 1, 0.1)
    dh = randn((rows, cols), dtype, rows + 2, 0.1)
    for k, gdt in enumerate((torch.float32, torch.bfloat16, None)):
        gain = None if gdt is None else randn((cols,), gdt, 3)
        rstd = F.fp4root_rmsnorm_quantize(h, gain, eps=1e-3, quantize=False).rstd
        e = dh if k != 1 else None
        dx, dgain = F.fp4root_rmsnorm_backward(dy, h, gain, rstd, dh=e)
        check_backward(dy, h, gain, rstd, e, dx, dgain, 1e-3)
        again, g2 = F.fp4root_rmsnorm_backward(dy, h, gain, rstd, dh=e)
        assert torch.equal(again, dx) and torch.equal(g2, dgain)


@pytest.mark.parametrize("rows,cols", [(2050, 2100), (2049, 4096), (4100, 1500), (2600, 5000), (70000, 40)])
def test_backward_of_many_rows(rows, cols):
    """More rows than workgroups, with 2 and 3 workgroups a CU and rows that share one."""
    h, dy = randn((rows, cols), torch.bfloat16, 61), randn((rows, cols), torch.bfloat16, 62)
    gain = randn((cols,), torch.float32, 63)
    rstd = F.fp4root_rmsnorm_quantize(h, gain, quantize=False).rstd
    dx, dgain = F.fp4root_rmsnorm_backward(dy, h, gain, rstd, dh=h)
    check_backward(dy, h, gain, rstd, h, dx, dgain, 1e-6)


def test_backward_against_differences():
    """The whole path in binary32 from the kernel's own forward values would be too coarse: the
    formula's loss in binary64, differenced in every direction of a small case."""
    rows, cols, eps = 3, 20, 1e-2
    h, dy = randn((rows, cols), torch.float32, 31), randn((rows, cols), torch.float32, 32)
    gain, dh = randn((cols,), torch.float32, 33), randn((rows, cols), torch.float32, 34)
    o = F.fp4root_rmsnorm_quantize(h, gain, eps=eps)
    dx, dgain = F.fp4root_rmsnorm_backward(dy, h, gain, o.rstd, dh=dh)

    def loss(hv, gv):
        y = hv / np.sqrt((hv * hv).mean(1, keepdims=True) + eps) * gv
        return (y * np64(dy)).sum() + (hv * np64(dh)).sum()
    h64, g64, s = np64(h), np64(gain), 1e-5
    for i in range(rows):
        for j in range(cols):
            d = np.zeros_like(h64)
            d[i, j] = s
            num = (loss(h64 + d, g64) - loss(h64 - d, g64)) / (2 * s)
            assert abs(num - float(dx[i, j])) <= 2e-5 * (1 + abs(num))
    for j in range(cols):
        d = np.zeros_like(g64)
        d[j] = s
        num = (loss(h64, g64 + d) - loss(h64, g64 - d)) / (2 * s)
        assert abs(num - float(dgain[j])) <= 2e-5 * (1 + abs(num))


@pytest.mark.parametrize("cols", [64, 200, 515, 4096, 8200, 16401])
def test_backward_strides_and_in_place(cols):
    buf = randn((9, 3 * cols + 5), torch.bfloat16, 35)
    h, dy, dh = buf[:, 1:1 + cols], buf[:, cols + 2:2 * cols + 2], buf[:, 2 * cols + 3:3 * cols + 3]
    gain = randn((cols,), torch.bfloat16, 36)
    rstd = F.fp4root_rmsnorm_quantize(h.contiguous(), gain, quantize=False).rstd
    dx, dgain = F.fp4root_rmsnorm_backward(dy.contiguous(), h.contiguous(), gain, rstd, dh=dh.contiguous())
    got, g2 = F.fp4root_rmsnorm_backward(dy, h, gain, rstd, dh=dh)
    assert torch.equal(got, dx) and torch.equal(g2, dgain)
    for target in (dh, dy, h):
        work = buf.clone()
        views = {id(v): work.as_strided(v.shape, v.stride(), v.storage_offset()) for v in (h, dy, dh)}
        a, b, c = views[id(h)], views[id(dy)], views[id(dh)]
        t = views[id(target)]
        out, g3 = F.fp4root_rmsnorm_backward(b, a, gain, rstd, dh=c, dx=t)
        assert out is t and torch.equal(t, dx) and torch.equal(g3, dgain)
        want = buf.clone()
        want.as_strided(target.shape, target.stride(), target.storage_offset()).copy_(dx)
        assert torch.equal(work, want)
    only, none = F.fp4root_rmsnorm_backward(dy, h, gain, rstd, want_dgain=False)
    assert none is None and torch.equal(only, F.fp4root_rmsnorm_backward(dy, h, gain, rstd)[0])


def test_graph_replay_and_streams():
    x, res = randn((33, 2000), torch.bfloat16, 40), randn((33, 2000), torch.bfloat16, 41)
    gain, dy = randn((2000,), torch.bfloat16, 42), randn((33, 2000), torch.bfloat16, 43)
    side = torch.cuda.Stream()

    def step(stream=None):
        o = F.fp4root_rmsnorm_quantize(x, gain, res, group=32, e8m0=True, stream=stream)
        return o, F.fp4root_rmsnorm_backward(dy, o.h, gain, o.rstd, dh=dy, stream=stream)
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        o, (dx, dgain) = step()
    for k in range(4):
        x.normal_(generator=gen(50 + k))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (o.codes, o.scales, o.rstd, o.h, dx, dgain)]
        e, (ex, eg) = step()
        assert all(torch.equal(a, b) for a, b in zip(got, (e.codes, e.scales, e.rstd, e.h, ex, eg)))
    want = step()
    torch.cuda.synchronize()
    s2 = torch.cuda.Stream()
    for _ in range(5):
        a, b = step(side), step(s2)
    torch.cuda.synchronize()
    for q in (a, b):
        assert torch.equal(q[0].codes, want[0].codes) and torch.equal(q[1][1], want[1][1])
