"""Host-side refusals of the gradient norm, clipping and RMS norm entry points (CPU only: the
pointers are never dereferenced, every call here fails before a launch or asks for sizes)."""
import ctypes
import math

import pytest
import torch

from paper_2607_04422_amd import fp4root as F

P = 0x100000          # fake device addresses, far apart
Q = 0x10000000
WS = 0x40000000
NAN, INF = math.nan, math.inf


def tensor(in_=P, out=Q, rows=4, cols=64, ld_in=64, ld_out=64, in_type=0, out_type=0):
    return F.Tensor(in_, out, rows, cols, ld_in, ld_out, in_type, out_type)


def array(*ts):
    return (F.Tensor * max(len(ts), 1))(*ts)


def norm(ts, count=None, kind=0, max_norm=1.0, eps=1e-6, total=Q, result=Q + 64, ws=WS, ws_bytes=1 << 20, norms=None):
    return F.load().fp4root_grad_norm(array(*ts), len(ts) if count is None else count, kind, max_norm, eps, total, norms,
                                      result, ws, ws_bytes, None)


def clip(*ts, coef=WS):
    return F.load().fp4root_clip_grads(array(*ts), len(ts), coef, None)


def test_norm_refusals():
    t = tensor()
    assert norm([t], count=-1) == -1
    assert norm([t], count=(1 << 20) + 1) == -1
    assert norm([t], kind=2) == -1
    for bad in (0.0, -1.0, NAN):
        assert norm([t], max_norm=bad) == -1
    for bad in (-1e-6, NAN, INF):
        assert norm([t], eps=bad) == -1
    assert norm([t], total=None) == -1
    assert norm([t], total=Q + 4) == -1
    assert norm([t], result=None) == -1
    assert norm([t], norms=Q + 2) == -1
    assert norm([t], ws=None) == -3
    assert norm([t], ws_bytes=F.load().fp4root_grad_norm_workspace(array(t), 1) - 1) == -3
    assert norm([tensor(in_type=3)]) == -1
    assert norm([tensor(rows=-1)]) == -2
    assert norm([tensor(cols=1 << 37)]) == -2
    assert norm([tensor(rows=1 << 20, cols=1 << 20, ld_in=1 << 20)]) == -2
    assert norm([tensor(ld_in=63)]) == -2
    assert norm([tensor(ld_in=1 << 40)]) == -2
    assert norm([tensor(in_=None)]) == -1
    assert norm([tensor(in_=P + 2)]) == -1
    assert norm([tensor(in_=P + 1, in_type=1)]) == -1
    assert norm([t, tensor(in_type=7)]) == -1        # every tensor is checked


def test_norm_workspace():
    lib = F.load()
    assert lib.fp4root_grad_norm_workspace(array(), 0) > 0
    assert lib.fp4root_grad_norm_workspace(array(tensor(ld_in=3)), 1) == 0
    assert lib.fp4root_grad_norm_workspace(array(tensor(rows=0, in_=None)), 1) > 0
    # at most 1024 partial sums a tensor
    big = lib.fp4root_grad_norm_workspace(array(tensor(rows=1, cols=1 << 36)), 1)
    assert big <= 5 * 256 + 1024 * 8


def test_clip_coef_refusals():
    lib = F.load()
    assert lib.fp4root_clip_coef(None, 0, 1.0, 0.0, P, None) == -1
    assert lib.fp4root_clip_coef(Q, 0, 1.0, 0.0, None, None) == -1
    assert lib.fp4root_clip_coef(Q, 5, 1.0, 0.0, P, None) == -1
    assert lib.fp4root_clip_coef(Q, 0, 0.0, 0.0, P, None) == -1


def test_clip_refuses_overlaps():
    """An output may be its own input and nothing else: workgroups run side by side."""
    assert clip(tensor(), coef=None) == -1
    assert clip(tensor(out=None)) == -1
    assert clip(tensor(out_type=9)) == -1
    assert clip(tensor(out=Q + 2)) == -1
    assert clip(tensor(ld_out=8)) == -2
    assert clip(tensor(out=P, out_type=1)) == -1                    # in place under another type
    assert clip(tensor(out=P, ld_out=128)) == -1                    # ... another stride
    assert clip(tensor(out=P + 64)) == -1                           # partly over itself
    one = tensor(out=P)
    assert clip(one, one) == -1                                     # listed twice
    assert clip(tensor(out=P), tensor(in_=P, out=Q)) == -1          # read while written
    assert clip(tensor(out=Q), tensor(in_=P, out=Q + 128)) == -1    # two outputs
    # columns 0..31 and 16..47 of one matrix with row stride 64
    a = tensor(in_=P, out=P, cols=32)
    assert clip(a, tensor(in_=P + 64, out=P + 64, cols=32)) == -1
    # wrapping into the next row's first columns
    assert clip(a, tensor(in_=P + 128 + 4, out=P + 128 + 4, cols=32)) == -1
    # a vector inside the matrix's columns
    assert clip(a, tensor(in_=P + 256, out=P + 256, rows=1, cols=8)) == -1


def rms(**kw):
    a = F.RmsNorm(x=P, gain=P + 0x80000, h=None, y=None, codes=Q, scales=Q + 0x80000, rstd=None, rows=4, cols=64,
                  ld_x=64, ld_residual=64, ld_h=64, ld_y=64, type=1, gain_type=1, group=0, scale_type=0, eps=1e-6)
    for k, v in kw.items():
        setattr(a, k, v)
    return F.load().fp4root_rmsnorm_quantize(ctypes.byref(a), None)


def test_rmsnorm_refusals():
    assert F.load().fp4root_rmsnorm_quantize(None, None) == -1
    for kw in (dict(type=3), dict(gain_type=2), dict(group=16), dict(group=-1), dict(scale_type=2), dict(eps=0.0),
               dict(eps=NAN), dict(eps=INF), dict(x=None), dict(scales=None), dict(codes=None),
               dict(codes=None, scales=None), dict(x=P + 1), dict(gain=P + 1), dict(rstd=Q + 0x90001),
               dict(scales=Q + 0x80002), dict(status=Q + 0x90002)):
        assert rms(**kw) == -1, kw
    for kw in (dict(cols=0), dict(cols=32769), dict(rows=-1), dict(ld_x=63), dict(residual=P + 0x40000, ld_residual=8),
               dict(h=Q + 0x40000, ld_h=32), dict(y=Q + 0x40000, ld_y=32), dict(ld_x=1 << 34)):
        assert rms(**kw) == -2, kw
    # outputs over inputs and over each other
    for kw in (dict(h=P, ld_h=80), dict(h=P + 2), dict(codes=P), dict(scales=P), dict(rstd=P), dict(codes=P + 0x80000),
               dict(h=Q), dict(h=P, y=P), dict(rstd=Q), dict(status=Q + 0x80004)):
        assert rms(**kw) == -1, kw
    assert rms(rows=0) == 0


def test_rmsnorm_backward_refusals():
    lib = F.load()
    need = lib.fp4root_rmsnorm_backward_workspace(4, 64)
    assert need >= 256
    assert lib.fp4root_rmsnorm_backward_workspace(4, 0) == 0
    assert lib.fp4root_rmsnorm_backward_workspace(4, 32769) == 0

    def call(dy=P, ld_dy=64, h=P + 0x10000, ld_h=64, dh=None, ld_dh=0, gain=P + 0x20000, rstd=P + 0x30000, dx=Q,
             ld_dx=64, dgain=Q + 0x10000, rows=4, cols=64, type_=1, gain_type=1, ws=WS, ws_bytes=1 << 20):
        return lib.fp4root_rmsnorm_backward(dy, ld_dy, h, ld_h, dh, ld_dh, gain, rstd, dx, ld_dx, dgain, rows, cols,
                                            type_, gain_type, ws, ws_bytes, None)
    for kw in (dict(dy=None), dict(h=None), dict(rstd=None), dict(dx=None), dict(type_=4), dict(gain_type=2),
               dict(dy=P + 1), dict(rstd=P + 0x30002), dict(dgain=Q + 0x10002), dict(dx=P + 2), dict(dx=P, ld_dx=128),
               dict(dx=P + 0x20000), dict(dgain=P + 0x30000), dict(dgain=Q + 4), dict(ws=Q), dict(ws=P)):
        assert call(**kw) == -1, kw
    for kw in (dict(cols=0), dict(cols=40000), dict(rows=-1), dict(ld_dy=63), dict(ld_h=1), dict(ld_dx=63),
               dict(dh=P + 0x50000, ld_dh=9)):
        assert call(**kw) == -2, kw
    assert call(ws=None) == -3
    assert call(ws_bytes=need - 1) == -3


def test_scaled_steps_refuse_a_misaligned_scale():
    lib = F.load()
    assert lib.fp4root_momentum_update_scaled(P, Q, 1, 64, 64, Q + 0x80000, Q + 0x90000, Q + 0xa0000, 0.9, 6, 0, 0,
                                              P + 2, WS, 1 << 20, None) == -1
    assert lib.fp4root_qadamw_update_scaled(P, P + 0x10000, None, 256, Q, Q + 0x1000, Q + 0x2000, Q + 0x3000, Q + 0x4000,
                                            Q + 0x5000, 1e-3, 0.1, 0.9, 0.95, 1e-8, 6, 0, 0, WS + 1, WS + 0x100, 1 << 20,
                                            None) == -1
    cfg, ns = F.RootConfig(0.01, 0.1, 0.9, 6, 0, 0), F.NsConfig(5, None, 7, 0.99, 1e-7, 0)
    assert lib.fp4root_root_step_scaled(None, 0, ctypes.byref(cfg), ctypes.byref(ns), WS + 1, WS, 1 << 30, None) == -1


def test_binding_refuses_cpu_tensors_and_bad_arguments():
    x = torch.zeros(4, 64)
    with pytest.raises(TypeError):
        F.GradClipper([x], 1.0)
    with pytest.raises(TypeError):
        F.fp4root_rmsnorm_quantize(x)
    with pytest.raises(TypeError):
        F.fp4root_rmsnorm_backward(x, x, None, torch.zeros(4))
    for bad in (0.0, -1.0, NAN):
        with pytest.raises(ValueError):
            F.GradClipper([], bad)
    with pytest.raises(ValueError):
        F.GradClipper([], 1.0, norm_type=1)
    with pytest.raises(ValueError):
        F.GradClipper([], 1.0, outputs=[x])


@pytest.mark.parametrize("view,want", [
    (lambda t: t, (1, 96, 96)), (lambda t: t[:, :, :4], (12, 4, 8)), (lambda t: t[:, 1:3], (3, 16, 32)),
    (lambda t: t.permute(2, 0, 1), (1, 96, 96)), (lambda t: t[0, :, :5].t(), (4, 5, 8)), (lambda t: t[:, 0, 0], (3, 1, 32)),
    (lambda t: t[1:1], (0, 0, 0)), (lambda t: t[2, 3, 7], (1, 1, 1)), (lambda t: t[..., ::2], (48, 1, 2))])
def test_rows_of_a_view(view, want):
    assert F._as_rows(view(torch.zeros(3, 4, 8)), "t") == want


def test_rows_of_refused_views():
    t = torch.zeros(3, 4, 8)
    for bad in (t[:, :2, :4], torch.zeros(1, 8).expand(4, 8), torch.zeros(40).as_strided((4, 8), (4, 1))):
        with pytest.raises(ValueError):
            F._as_rows(bad, "t")
