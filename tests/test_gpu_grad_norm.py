"""Gradient norm and clipping (fp4root_grad_list_*, fp4root_grad_norm,
fp4root_clip_coef, fp4root_clip_grads) and the
optimizer steps that read gradients through the clipping coefficient.

Tolerances.  A total is a binary64 sum of exact squares: any order of n additions is within
n 2^-53 of the exact one.  A norm rounds its root to binary32 once more (2^-24), the root itself
to binary64.  Maxima, clipped elements and the steps are compared bit for bit."""
import math

import numpy as np
import pytest
import torch

from tests.gpu_util import need_gpu

pytestmark = pytest.mark.gpu

F = None
TYPES = [torch.float32, torch.bfloat16, torch.float16]
HALF = 2.0 ** -24


def setup_module():
    global F
    need_gpu()
    from paper_2607_04422_amd import fp4root
    F = fp4root


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def make(shapes, dtype, seed=0):
    g = gen(seed)
    return [(torch.randn(s, generator=g, device="cuda") * 0.1).to(dtype) for s in shapes]


def totals(grads, kind=2):
    """Each tensor's sum of squares or maximum, in binary64."""
    vals = [g.detach().cpu().double().numpy().reshape(-1) for g in grads]
    if kind == 2:
        return [math.fsum((v * v).tolist()) for v in vals]
    return [float(np.max(np.abs(v))) if v.size else 0.0 for v in vals]


def check(c, grads, kind=2):
    each = totals(grads, kind)
    n = sum(g.numel() for g in grads)
    total = math.fsum(each) if kind == 2 else max(each, default=0.0)
    tol = (n + 2) * 2.0 ** -53 if kind == 2 else 0.0
    assert abs(float(c.total) - total) <= tol * total
    for got, want in zip(c.norms.tolist(), each):
        want = math.sqrt(want) if kind == 2 else want
        assert abs(got - want) <= (HALF * 1.001 + tol) * want + 2.0 ** -150
    norm = math.sqrt(total) if kind == 2 else total
    assert abs(float(c.total_norm) - norm) <= (HALF * 1.001 + tol) * norm + 2.0 ** -150
    want = min(1.0, c.max_norm / (norm + c.eps)) if norm + c.eps else 1.0
    # a coefficient below 2^-126 is a multiple of 2^-149, off by half of that at most
    assert abs(float(c.coef) - want) <= (HALF * 1.001 + tol) * want + 2.0 ** -150


LISTS = {
    "one": [(1,)],
    "odd": [(1,), (7,), (4097,), (33, 515), (65537,)],
    "ragged_130": [(1 + 37 * i,) for i in range(130)],
    "exactly_64": [(17, 5)] * 64,
    "parts": [(1 << 18,), ((1 << 18) + 1,), (3, 1 << 18)],
    "empty": [(0,), (5, 0), (3,), (0,)],
    "all_empty": [(0,)],
    "none": [],
}


@pytest.mark.parametrize("kind", [2, math.inf])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("name", list(LISTS))
def test_norm_and_clip(name, dtype, kind):
    grads = make(LISTS[name], dtype)
    for max_norm in (1e-2, 1e6, math.inf):
        outs = [torch.full_like(g, 7.0, dtype=torch.float32) for g in grads]
        c = F.GradClipper(grads, max_norm, outputs=outs, norm_type=kind)
        assert c.status() == 0 and float(c.total) == 0.0
        c()
        check(c, grads, kind)
        for g, o in zip(grads, outs):
            assert torch.equal(o, g.float() * c.coef)
        assert c.status() == 0


def test_mixed_types_and_many_tensors():
    """Types side by side in one list, and more tensors than one workgroup joins."""
    for n in (15, 16, 17, 47, 48, 49, 63, 64, 65, 1100):
        grads = [make([(1 + 61 * (i % 23), 3)], TYPES[i % 3], i)[0] for i in range(n)]
        want = [g.clone() for g in grads]
        for kind in (2, math.inf):
            c = F.GradClipper(grads, 0.3, norm_type=kind, outputs=[torch.zeros_like(g, dtype=torch.float32) for g in grads])
            for g, o in zip(want, c()):
                assert torch.equal(o, g.float() * c.coef)
            check(c, want, kind)


@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("dtype", TYPES)
def test_clip_types(dtype, out):
    grads = make([(129, 67), (8,), (4099,)], dtype, 3)
    if dtype == torch.float32:
        grads[0][5, 6] = 1e5           # past float16 after clipping by 0.9
    outs = [torch.empty_like(g, dtype=out) for g in grads]
    c = F.GradClipper(grads, 0.9 * float(torch.cat([g.float().reshape(-1) for g in grads]).norm()), outputs=outs)
    c()
    assert 0.8 < float(c.coef) < 1
    for g, o in zip(grads, outs):
        assert torch.equal(o, (g.float() * c.coef).to(out))
    assert bool(torch.isinf(outs[0].float()).any()) == (dtype == torch.float32 and out == torch.float16)


@pytest.mark.parametrize("dtype", TYPES)
def test_clip_in_place_and_untouched(dtype):
    """Views of one buffer: columns, rows, a transpose and unaligned runs, in place; what lies
    between them stays."""
    buf = make([(400, 130)], dtype, 4)[0]
    grads = [buf[:100, :65], buf[:100, 65:], buf[100:200, 3:40], buf[200:300, 1:9].t(), buf[301:303].reshape(-1)[3:250],
             buf[310:, ::2]]
    keep = buf.clone()
    mask = torch.zeros_like(buf, dtype=torch.bool)
    for m in (mask[:100, :65], mask[:100, 65:], mask[100:200, 3:40], mask[200:300, 1:9].t(),
              mask[301:303].reshape(-1)[3:250], mask[310:, ::2]):
        m.fill_(True)
    want = [g.clone() for g in grads]
    c = F.GradClipper(grads, 1.0)
    c()
    check(c, want)
    for g, w in zip(grads, want):
        assert torch.equal(g, (w.float() * c.coef).to(dtype))
    assert torch.equal(buf[~mask], keep[~mask])
    # a norm below max_norm: nothing changes
    before = buf.clone()
    c2 = F.GradClipper(grads, 1e6)
    c2()
    assert float(c2.coef) == 1.0 and torch.equal(buf, before)


def test_rows_beside_contiguous():
    grads = [make([(50, 90)], torch.bfloat16, 5)[0][:, 7:70], make([(50, 63)], torch.bfloat16, 6)[0]]
    wide = torch.zeros((50, 200), device="cuda")
    outs = [torch.zeros((50, 63), device="cuda"), wide[:, 100:163]]
    c = F.GradClipper(grads, 0.5, outputs=outs)
    c()
    for g, o in zip(grads, outs):
        assert torch.equal(o, g.float() * c.coef)
    assert float(wide[:, :100].abs().max()) == 0 and float(wide[:, 163:].abs().max()) == 0
    for bad in (torch.zeros((63, 50), device="cuda").t(), torch.zeros((50, 64), device="cuda")):
        with pytest.raises(ValueError):
            F.GradClipper(grads[:1], 0.5, outputs=[bad])
    with pytest.raises(F.Fp4RootError):
        F.GradClipper([grads[1], grads[1]], 0.5)
    with pytest.raises(ValueError):
        F.GradClipper(grads, 0.5, outputs=outs, measure_only=True)
    twice = F.GradClipper([grads[1], grads[1]], 0.5, measure_only=True)
    twice.norm()
    check(twice, [grads[1], grads[1]])
    with pytest.raises(F.Fp4RootError):
        twice.scale()


def test_extremes_of_the_type():
    """Squares past binary32 both ways, subnormals, and a sum dominated by one element."""
    f = lambda *v: torch.tensor(v, device="cuda")      # noqa: E731
    for grads in ([f(3e38, 3e38, -3e38)], [f(1e-40, 2e-45)], [f(1e30), f(1e-30)], [torch.zeros(9, device="cuda")]):
        for kind in (2, math.inf):
            c = F.GradClipper(grads, 1.0, norm_type=kind)
            c.norm()
            if kind == 2 and float(grads[0].abs().max()) > 1e38:
                assert float(c.total) == pytest.approx(27e76, rel=1e-6) and math.isinf(float(c.total_norm))
                assert float(c.coef) == pytest.approx(1 / math.sqrt(27e76), rel=1e-6)
            else:
                check(c, grads, kind)


@pytest.mark.parametrize("kind", [2, math.inf])
def test_non_finite(kind):
    for at, where in ((0, 0), (70, 5), (129, 4000)):
        for bad in (math.nan, math.inf, -math.inf):
            grads = make([(4097,)] * 130, torch.bfloat16, 7)
            grads[at][where] = bad
            outs = [torch.zeros(4097, device="cuda") for _ in grads]
            c = F.GradClipper(grads, 1.0, outputs=outs, norm_type=kind)
            c()
            assert c.status() == -4
            if math.isnan(bad):
                assert math.isnan(float(c.total_norm)) and math.isnan(float(c.coef)) and math.isnan(c.norms[at].item())
                assert torch.isnan(outs[0]).all()
            else:
                assert math.isinf(float(c.total_norm)) and float(c.coef) == 0.0 and math.isinf(c.norms[at].item())
                assert math.isnan(outs[at][where].item()) and float(outs[at][where - 1].abs()) == 0.0
            assert math.isfinite(c.norms[at - 1].item())
            grads[at][where] = 0.0
            c()
            assert c.status() == 0
            check(c, grads, kind)


def test_same_bits_beside_other_tensors_and_again():
    grads = make([(1 << 20,), (511, 1031), (77,)], torch.float32, 8)
    alone = [F.GradClipper([g], 1.0) for g in grads]
    for a in alone:
        a.norm()
    many = F.GradClipper(make([(3000,)] * 70, torch.bfloat16, 9) + grads, 1.0)
    many.norm()
    first = many.total.clone()
    for i, a in enumerate(alone):
        assert float(many.norms[70 + i]) == float(a.norms[0])
    for _ in range(5):
        many.norm()
        assert torch.equal(many.total, first)


def test_far_rows_and_long_tensors():
    """Offsets past 2^32 elements, and parts past the first 1024 sizes."""
    n = (1 << 32) + 11
    big = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    big[-1], big[0], big[1 << 31] = 3.0, 4.0, 12.0
    c = F.GradClipper([big], 1.0)
    c()
    assert float(c.total) == 169.0 and float(c.total_norm) == 13.0
    assert [float(big[i]) for i in (-1, 0, 1 << 31)] == \
        [float((torch.tensor(v) * c.coef.cpu()).bfloat16()) for v in (3.0, 4.0, 12.0)]
    rows = big[:3 * (1 << 30)].view(3, 1 << 30)[:, 5:16]
    rows.copy_(torch.arange(33, device="cuda").view(3, 11))
    c = F.GradClipper([rows], 1e9)
    c.norm()
    assert float(c.total) == sum(i * i for i in range(33))


def test_all_reduce_between():
    """Ranks add `total` before the coefficient: two shards against the whole."""
    whole = make([(999, 33), (4096,)], torch.float32, 10)
    for kind in (2, math.inf):
        ref = F.GradClipper(whole, 0.5, norm_type=kind)
        ref.norm()
        shards = [F.GradClipper([whole[0][:500], whole[1][:7]], 0.5, norm_type=kind,
                                outputs=[torch.empty_like(whole[0][:500]), torch.empty_like(whole[1][:7])]),
                  F.GradClipper([whole[0][500:], whole[1][7:]], 0.5, norm_type=kind)]
        for s in shards:
            s.norm()
        both = torch.stack([s.total for s in shards])
        total = both.sum(0) if kind == 2 else both.amax(0)
        for s in shards:
            s.total.copy_(total)
            s.recoef()
            assert float(s.total_norm) == pytest.approx(float(ref.total_norm), rel=2 ** -23)
            assert float(s.coef) == pytest.approx(float(ref.coef), rel=2 ** -23)
        got = shards[0].scale()
        assert torch.equal(got[0], whole[0][:500] * shards[0].coef)


def test_graph_replay_and_streams():
    grads = make([(4096, 33), (515,), (1 << 20,)], torch.bfloat16, 11)
    outs = [torch.empty_like(g, dtype=torch.float32) for g in grads]
    c = F.GradClipper(grads, 0.7, outputs=outs)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        c()
    for k in range(4):
        for g in grads:
            g.normal_(generator=gen(100 + k)).mul_(0.01 * (k + 1))
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs], c.total.clone(), c.result.clone()
        eager = F.GradClipper(grads, 0.7, outputs=[torch.empty_like(o) for o in outs])
        e = eager()
        assert torch.equal(got[1], eager.total) and torch.equal(got[2], eager.result)
        assert all(torch.equal(a, b) for a, b in zip(got[0], e))
    # two clippers at once on two streams
    other = make([(1 << 20,)] * 8, torch.float32, 12)
    d = F.GradClipper(other, 0.1)
    want = (F.GradClipper(other, 0.1).norm().item(), eager.total_norm.item())
    s2 = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(10):
        d.norm(side)
        eager.norm(s2)
    torch.cuda.synchronize()
    assert (d.total_norm.item(), eager.total_norm.item()) == want


def test_function_in_place():
    grads = make([(100, 7), (3,)], torch.float32, 13)
    want = [g.clone() for g in grads]
    other = [g.clone() for g in grads]
    norm = F.fp4root_clip_grads(grads, 0.25)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = F.fp4root_clip_grads(other, 0.25, stream=side)
    torch.cuda.synchronize()
    assert float(again) == float(norm) and all(torch.equal(a, b) for a, b in zip(other, grads))
    ref = torch.cat([w.reshape(-1) for w in want]).double().norm()
    assert float(norm) == pytest.approx(float(ref), rel=1e-6)
    coef = torch.tensor(min(1.0, 0.25 / (float(ref) + 1e-6)), dtype=torch.float32)
    for g, w in zip(grads, want):
        assert torch.allclose(g, w * coef.cuda(), rtol=2 ** -22, atol=0)


def test_function_captured():
    """The one-call form allocates and builds its list inside the capture."""
    grads = make([(100, 7), (70000,)], torch.bfloat16, 33)
    outs = [torch.zeros_like(g, dtype=torch.float32) for g in grads]
    F.fp4root_clip_grads(grads, 0.25, outputs=outs)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        norm = F.fp4root_clip_grads(grads, 0.25, outputs=outs)
    for k in range(3):
        grads[1].mul_(1.5)
        graph.replay()
        torch.cuda.synchronize()
        got = float(norm), [o.clone() for o in outs]
        assert float(F.fp4root_clip_grads(grads, 0.25, outputs=outs)) == got[0]
        assert all(torch.equal(a, b) for a, b in zip(outs, got[1]))


# ---- the steps that read gradients times the coefficient ----

FLAGS = [6, 22, 0]


@pytest.mark.parametrize("flags", FLAGS)
def test_scaled_momentum_equals_clipping_first(flags):
    g = make([(3, 48, 64)], torch.float32, 14)[0]
    scale = torch.tensor([0.3712], device="cuda")
    a, b = F.MomentumState(3, 48, 64), F.MomentumState(3, 48, 64)
    for t in range(3):
        ma = F.fp4root_momentum_update(g, a, 0.9, t, flags, seed=4, grad_scale=scale)
        mb = F.fp4root_momentum_update(g * scale, b, 0.9, t, flags, seed=4)
        assert torch.equal(ma, mb) and torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales)
        assert torch.equal(a.tensor_scale, b.tensor_scale)
        g = g.roll(1, 0) * 1.5
    # in place, where m is g
    m = g.clone()
    F.fp4root_momentum_update(m, a, 0.9, 3, flags, seed=4, m=m, grad_scale=scale)
    assert torch.equal(m, F.fp4root_momentum_update(g * scale, b, 0.9, 3, flags, seed=4))


@pytest.mark.parametrize("flags", FLAGS)
def test_scaled_qadamw_equals_clipping_first(flags):
    n = 256 * 37
    w0 = make([(n,)], torch.bfloat16, 15)[0]
    wa, wb = w0.clone(), w0.clone()
    a, b = F.QAdamWState(n, keep_m=True), F.QAdamWState(n, keep_m=True)
    scale = torch.tensor(0.0625 * 1.7, device="cuda")
    for t in range(3):
        g = make([(n,)], torch.float32, 16 + t)[0]
        F.fp4root_qadamw_update(wa, g, a, t, 1e-3, flags=flags, seed=5, grad_scale=scale)
        F.fp4root_qadamw_update(wb, g * scale, b, t, 1e-3, flags=flags, seed=5)
        for name in ("m", "m_codes", "m_scales", "m_tensor_scale", "v_codes", "v_scales", "v_means"):
            assert torch.equal(getattr(a, name), getattr(b, name)), (t, name)
        assert torch.equal(wa, wb)
    # a coefficient that is not a number reaches the status
    F.fp4root_qadamw_update(wa, g, a, 3, 1e-3, flags=flags, seed=5, grad_scale=torch.tensor(math.nan, device="cuda"))
    assert F.fp4root_device_status(a.ws) == -4


def test_root_step_with_max_norm_equals_clipping_first():
    shapes = [(64, 128), (128, 64), (64, 128), (32, 32)]
    grads = make(shapes, torch.float32, 20)
    ws = make(shapes, torch.bfloat16, 21)
    wa, wb = [w.clone() for w in ws], [w.clone() for w in ws]
    ga, gb = grads, [g.clone() for g in grads]
    a = F.RootStep(wa, ga, 0.02, max_norm=0.5, seed=3)
    b = F.RootStep(wb, gb, 0.02, seed=3)
    for t in range(2):
        for x, y in zip(ga, gb):
            y.copy_(x)
        keep = [g.clone() for g in ga]
        a(t)
        c = F.GradClipper(gb, 0.5)
        c()
        assert float(c.coef) < 1 and float(c.total_norm) == float(a.clipper.total_norm)
        b(t)
        assert all(torch.equal(x, y) for x, y in zip(wa, wb))
        assert all(torch.equal(x.codes, y.codes) for x, y in zip(a.states, b.states))
        assert all(torch.equal(x, y) for x, y in zip(ga, keep))      # the gradients stay as they were
        assert a.status() == 0
        for g in ga:
            g.mul_(1.3).add_(0.01)
    with pytest.raises(ValueError):
        a(2, grad_scale=c.coef)
    with pytest.raises(ValueError):
        b(2, grad_scale=torch.ones(2, device="cuda"))
