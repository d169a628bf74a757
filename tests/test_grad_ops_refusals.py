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


def init(*ts, count=None, mem=WS, mem_bytes=1 << 20):
    """An init that has to fail: what would pass the checks has no GPU to run on."""
    out = F.GradList()
    rc = F.load().fp4root_grad_list_init(ctypes.byref(out), array(*ts), len(ts) if count is None else count, mem, mem_bytes,
                                         None)
    assert out.mem is None
    return rc


def test_list_refusals():
    t = tensor()
    assert F.load().fp4root_grad_list_init(None, array(t), 1, WS, 1 << 20, None) == -1
    assert init(t, count=-1) == -1
    assert init(t, count=(1 << 20) + 1) == -1
    assert init(t, mem=None) == -3
    assert init(t, mem=WS + 128) == -3
    assert init(t, mem_bytes=F.load().fp4root_grad_list_size(array(t), 1) - 1) == -3
    for bad, rc in ((dict(in_type=3), -1), (dict(rows=-1), -2), (dict(cols=1 << 37), -2),
                    (dict(rows=1 << 20, cols=1 << 20, ld_in=1 << 20), -2), (dict(ld_in=63), -2), (dict(ld_in=1 << 40), -2),
                    (dict(in_=None), -1), (dict(in_=P + 2), -1), (dict(in_=P + 1, in_type=1), -1),
                    (dict(out=None, in_=None), -1)):
        assert init(tensor(**bad)) == rc, bad
        assert init(t, tensor(**bad)) == rc, bad             # every tensor is checked
        assert F.load().fp4root_grad_list_size(array(tensor(**bad)), 1) == 0
    assert init(t, tensor(in_=P + 0x10000, out=None)) == -1  # outputs for all or for none


def test_list_size():
    lib = F.load()
    assert lib.fp4root_grad_list_size(array(), 0) > 0
    assert lib.fp4root_grad_list_size(array(tensor(rows=0, in_=None, out=None)), 1) > 0
    # at most 1024 parts a tensor
    big = lib.fp4root_grad_list_size(array(tensor(rows=1, cols=1 << 36, out=None)), 1)
    assert big <= 6 * 256 + 1024 * 16


def test_norm_refusals():
    lib = F.load()
    good = F.GradList(WS, 3, 5, 1)

    def norm(lst=good, kind=0, max_norm=1.0, eps=1e-6, total=Q, result=Q + 64, norms=None):
        return lib.fp4root_grad_norm(ctypes.byref(lst) if lst else None, kind, max_norm, eps, total, norms, result, None)
    for bad in (0.0, -1.0, NAN):
        assert norm(max_norm=bad) == -1
    for bad in (-1e-6, NAN, INF):
        assert norm(eps=bad) == -1
    for kw in (dict(lst=None), dict(lst=F.GradList()), dict(lst=F.GradList(WS + 4, 3, 5, 1)), dict(lst=F.GradList(WS, 3, 2, 1)),
               dict(lst=F.GradList(WS, 3, 4000, 1)), dict(kind=2), dict(total=None), dict(total=Q + 4), dict(result=None),
               dict(norms=Q + 2)):
        assert norm(**kw) == -1, kw
    for lst, coef in ((good, None), (good, Q + 2), (F.GradList(WS, 3, 5, 0), Q), (F.GradList(), Q)):
        assert lib.fp4root_clip_grads(ctypes.byref(lst), coef, None) == -1


def test_clip_coef_refusals():
    lib = F.load()
    assert lib.fp4root_clip_coef(None, 0, 1.0, 0.0, P, None) == -1
    assert lib.fp4root_clip_coef(Q, 0, 1.0, 0.0, None, None) == -1
    assert lib.fp4root_clip_coef(Q, 5, 1.0, 0.0, P, None) == -1
    assert lib.fp4root_clip_coef(Q, 0, 0.0, 0.0, P, None) == -1


def test_clip_refuses_overlaps():
    """An output may be its own input and nothing else: workgroups run side by side."""
    assert init(tensor(out_type=9)) == -1
    assert init(tensor(out=Q + 2)) == -1
    assert init(tensor(ld_out=8)) == -2
    assert init(tensor(out=P, out_type=1)) == -1                    # in place under another type
    assert init(tensor(out=P, ld_out=128)) == -1                    # ... another stride
    assert init(tensor(out=P + 64)) == -1                           # partly over itself
    one = tensor(out=P)
    assert init(one, one) == -1                                     # listed twice
    assert init(tensor(out=P), tensor(in_=P, out=Q)) == -1          # read while written
    assert init(tensor(out=Q), tensor(in_=P, out=Q + 128)) == -1    # two outputs
    # columns 0..31 and 16..47 of one matrix with row stride 64
    a = tensor(in_=P, out=P, cols=32)
    assert init(a, tensor(in_=P + 64, out=P + 64, cols=32)) == -1
    # wrapping into the next row's first columns
    assert init(a, tensor(in_=P + 128 + 4, out=P + 128 + 4, cols=32)) == -1
    # a vector inside the matrix's columns
    assert init(a, tensor(in_=P + 256, out=P + 256, rows=1, cols=8)) == -1


def rms(**kw):
    a = F.RmsNorm(x=P, gain=P + 0x80000, h=None, y=None, codes=Q, scales=Q + 0x80000, rstd=None, rows=4, cols=64,
                  ld_x=64, ld_residual=64, ld_h=64, ld_y=64, type=1, gain_type=1, group=0, scale_type=0, eps=1e-6)
    for k, v in kw.items():
        setattr(a, k, v)
    return F.load().fp4root_rmsnorm_quantize(ctypes.byref(a), None)


def test_rmsnorm_refusals():
    assert F.load().fp4root_rmsnorm_quantize(None, None) == -1
    for kw in (dict(type=3), dict(gain_type=2), dict(group=16), dict(group=-1), dict(scale_type=2), dict(eps=0.0),
               dict(eps=1e-39), dict(eps=NAN), dict(eps=INF), dict(x=None), dict(scales=None), dict(codes=None),
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


def test_row_of_a_thread_by_multiplication():
    """The kernels divide a thread's number by the threads a row takes through 2^20 over them,
    rounded up, in 32 bits."""
    for tpr in range(64, 1025, 64):
        inverse = -(-(1 << 20) // tpr)
        for t in range(1024):
            assert (t * inverse) >> 20 == t // tpr and t * inverse < 1 << 32


def test_a_stream_of_another_gpu_is_refused():
    class Stream:
        device, cuda_stream = torch.device("cuda", 1), 7
    assert F._launch_stream(torch.device("cuda", 1), Stream()) == 7
    with pytest.raises(ValueError):
        F._launch_stream(torch.device("cuda", 0), Stream())
