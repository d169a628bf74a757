"""A training step's operators in a row: the 8-bit norm before a quantized projection, the
gradients of both, the global norm over them, and the two optimizer steps that read them through
its coefficient; eagerly, and captured into a graph beside eager work."""
import numpy as np
import pytest
import torch

from tests.gpu_util import need_gpu

pytestmark = pytest.mark.gpu

F = None
ROWS, COLS, OUT = 96, 512, 64


def setup_module():
    global F
    need_gpu()
    from paper_2607_04422_amd import fp4root
    F = fp4root


class Net:
    """y = E4M3(norm(x + r) gain) W^T with a gradient of ones / rows on y; W by the Root step, gain
    by the quantized AdamW, both under one global norm."""

    def __init__(self, max_norm):
        g = torch.Generator(device="cuda").manual_seed(3)
        rnd = lambda *s: torch.randn(s, generator=g, device="cuda")      # noqa: E731
        self.x, self.r = rnd(ROWS, COLS).bfloat16(), rnd(ROWS, COLS).bfloat16()
        self.target = rnd(ROWS, OUT)
        self.w, self.gain = (rnd(OUT, COLS) * 0.05).bfloat16(), (1 + 0.1 * rnd(COLS)).bfloat16()
        self.dw, self.dgain = torch.zeros(OUT, COLS, device="cuda"), torch.zeros(COLS, device="cuda")
        self.clip = F.GradClipper([self.dw, self.dgain], max_norm, measure_only=True)
        self.root = F.RootStep([self.w], [self.dw], 0.02, seed=1)
        self.adam = F.QAdamWState(COLS)
        self.out = None

    def grads(self):
        o = F.fp4root_rmsnorm_quantize(self.x, self.gain, self.r, eps=1e-5, group=32, e8m0=True, out=self.out)
        scale = torch.exp2(o.scales.float() - 127.0).repeat_interleave(32, 1)
        q = o.codes.view(torch.float8_e4m3fn).float() * scale
        dy_out = (q @ self.w.float().t().contiguous() - self.target) / ROWS
        self.dw.copy_(dy_out.t().contiguous() @ q)
        dq = (dy_out @ self.w.float()).bfloat16()
        dx, _ = F.fp4root_rmsnorm_backward(dq, o.h, self.gain, o.rstd, dgain=self.dgain)
        return o, q, dq, dx

    def step(self, t):
        got = self.grads()
        self.clip.norm()
        self.root(t, grad_scale=self.clip.coef)
        F.fp4root_qadamw_update(self.gain, self.dgain, self.adam, t, 1e-2, seed=2, grad_scale=self.clip.coef)
        return got


def test_gradients_and_norm_of_the_chain():
    net = Net(0.01)
    o, q, dq, dx = net.grads()
    net.clip.norm()
    x64 = lambda t: t.double().cpu().numpy()      # noqa: E731
    h = x64((net.x.float() + net.r.float()).bfloat16())
    rstd = 1 / np.sqrt((h * h).mean(1, keepdims=True) + 1e-5)
    y = h * rstd * x64(net.gain)
    # a code is within 2^-4 of its value, or half the smallest step, 2^-10, of its scale
    scale = 2.0 ** (x64(o.scales) - 127).repeat(32, 1)
    assert np.all(np.abs(x64(q) - y) <= 2.0 ** -4 * np.abs(y) * (1 + 2.0 ** -20) + 2.0 ** -10 * scale)
    d = x64(dq)
    dgain = (d * h * rstd).sum(0)
    assert np.all(np.abs(x64(net.dgain) - dgain) <= 66 * 2.0 ** -24 * np.abs(d * h * rstd).sum(0))
    g = d * x64(net.gain)
    want = rstd * (g - h * rstd * (g * h * rstd).mean(1, keepdims=True))
    size = rstd * (np.abs(g) + np.abs(h * rstd) * np.abs(g * h * rstd).mean(1, keepdims=True))
    assert np.all(np.abs(x64(dx) - want) <= 2.0 ** -8 * np.abs(want) + 72 * 2.0 ** -24 * size)
    norm = np.sqrt((x64(net.dw) ** 2).sum() + (x64(net.dgain) ** 2).sum())
    assert abs(float(net.clip.total_norm) - norm) <= 2.0 ** -23 * norm
    assert float(net.clip.coef) < 1


def test_steps_equal_clipping_first():
    a, b = Net(0.01), Net(0.01)
    both = F.GradClipper([b.dw, b.dgain], 0.01)
    for t in range(3):
        a.step(t)
        b.grads()
        both()
        b.root(t)
        F.fp4root_qadamw_update(b.gain, b.dgain, b.adam, t, 1e-2, seed=2)
        assert torch.equal(a.w, b.w) and torch.equal(a.gain, b.gain)
        assert torch.equal(a.adam.v_codes, b.adam.v_codes) and torch.equal(a.root.states[0].codes, b.root.states[0].codes)
    assert a.root.status() == 0 and F.fp4root_device_status(a.adam.ws) == 0


def test_captured_step_replays_like_eager_ones():
    a, b = Net(0.01), Net(0.01)
    a.out = a.grads()[0]
    a.step(1)
    b.step(1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a.step(1)
    b.step(1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        a.step(1)
    for _ in range(4):
        a.x.mul_(0.9)
        b.x.mul_(0.9)
        graph.replay()
        torch.cuda.synchronize()
        b.step(1)
        assert torch.equal(a.dgain, b.dgain) and torch.equal(a.dw, b.dw)
        assert torch.equal(a.w, b.w) and torch.equal(a.gain, b.gain)
