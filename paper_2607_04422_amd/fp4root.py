"""ctypes binding of libfp4root.so (argument marshalling only).

Every function here checks its tensors, passes raw device pointers, sizes and
the current HIP stream to the C entry point of the same name, and raises
``Fp4RootError`` on a non-zero return code.  Device memory for outputs and the
workspace comes from PyTorch; all computation happens in the library's
kernels.  There is no CPU path: without the built library or a GPU every call
raises.
"""
from __future__ import annotations

import ctypes
import os
import re
from typing import NamedTuple, Optional

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libfp4root.so")
HEADER = os.path.join(os.path.dirname(HERE), "include", "fp4root.h")

OK = 0
F_CLIP = 1
F_HADAMARD = 2
F_ADAPTIVE46 = 4
F_BF16_PATH = 8
F_STOCHASTIC = 16
F_FP32_ACCUM = 32   # products accumulate in binary32 (MFMA order) instead of exactly
F_DEFAULT = 7


class Fp4RootError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {status_string(code)} ({code})")


class Matrix(ctypes.Structure):
    _fields_ = [("in_", ctypes.c_void_p), ("out", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("cols", ctypes.c_int64), ("ld_in", ctypes.c_int64), ("ld_out", ctypes.c_int64)]


class NsConfig(ctypes.Structure):
    _fields_ = [("steps", ctypes.c_int32), ("coeffs", ctypes.POINTER(ctypes.c_float)),
                ("flags", ctypes.c_uint32), ("clip_quantile", ctypes.c_float),
                ("eps", ctypes.c_float), ("seed", ctypes.c_uint64)]


class Param(ctypes.Structure):
    _fields_ = [("w", ctypes.c_void_p), ("g", ctypes.c_void_p), ("m", ctypes.c_void_p),
                ("m_codes", ctypes.c_void_p), ("m_scales", ctypes.c_void_p), ("m_tensor_scale", ctypes.c_void_p),
                ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("scale", ctypes.c_float)]


class RootConfig(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_float), ("wd", ctypes.c_float), ("beta", ctypes.c_float),
                ("momentum_flags", ctypes.c_uint32), ("momentum_seed", ctypes.c_uint64), ("step", ctypes.c_int32)]


FLOAT32, BFLOAT16, FLOAT16 = 0, 1, 2
NORM_L2, NORM_MAX = 0, 1
SCALE_FP32, SCALE_E8M0 = 0, 1
_TYPES = {torch.float32: FLOAT32, torch.bfloat16: BFLOAT16, torch.float16: FLOAT16}
_GAIN_TYPES = {torch.float32: FLOAT32, torch.bfloat16: BFLOAT16}


class Tensor(ctypes.Structure):
    _fields_ = [("in_", ctypes.c_void_p), ("out", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("cols", ctypes.c_int64), ("ld_in", ctypes.c_int64), ("ld_out", ctypes.c_int64),
                ("in_type", ctypes.c_int32), ("out_type", ctypes.c_int32)]


class GradList(ctypes.Structure):
    _fields_ = [("mem", ctypes.c_void_p), ("count", ctypes.c_int64), ("parts", ctypes.c_int64),
                ("flags", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class RmsNorm(ctypes.Structure):
    _fields_ = [(name, ctypes.c_void_p) for name in
                ("x", "residual", "gain", "h", "y", "codes", "scales", "rstd", "status")] + \
               [(name, ctypes.c_int64) for name in ("rows", "cols", "ld_x", "ld_residual", "ld_h", "ld_y")] + \
               [(name, ctypes.c_int32) for name in ("type", "gain_type", "group", "scale_type")] + \
               [("eps", ctypes.c_double)]


class NsTrace(ctypes.Structure):
    _fields_ = [(name, ctypes.c_void_p) for name in (
        "qx_codes", "qx_scales", "qx_sg", "qxt_codes", "qxt_scales", "qxt_sg", "A",
        "qa_codes", "qa_scales", "qa_sg", "B", "qb_codes", "qb_scales", "qb_sg")]


_lib = None


def load(path: str = None) -> ctypes.CDLL:
    """Load the library (once): `path`, else $FP4ROOT_LIBRARY, else the in-tree build.
    Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    path = path or os.environ.get("FP4ROOT_LIBRARY") or LIB_PATH
    if not os.path.exists(path):
        raise RuntimeError(f"libfp4root.so not built at {path}; run __graft_entry__.build()")
    lib = ctypes.CDLL(path)
    i64, u32, u64, f32, vp, i32 = (ctypes.c_int64, ctypes.c_uint32, ctypes.c_uint64,
                                   ctypes.c_float, ctypes.c_void_p, ctypes.c_int32)
    sz, f64 = ctypes.c_size_t, ctypes.c_double
    lib.fp4root_quantize_workspace.argtypes = [i64, i64, i64, u32]
    lib.fp4root_quantize_workspace.restype = sz
    lib.fp4root_ns_step_workspace.argtypes = [i64, i64, i64, u32]
    lib.fp4root_ns_step_workspace.restype = sz
    lib.fp4root_orthogonalize_workspace.argtypes = [ctypes.POINTER(Matrix), i64, ctypes.POINTER(NsConfig)]
    lib.fp4root_orthogonalize_workspace.restype = sz
    lib.fp4root_quantize.argtypes = [vp, i64, i64, i64, i64, i64, ctypes.c_int, u32, f32, u64, i32,
                                     vp, vp, vp, vp, vp, sz, vp]
    lib.fp4root_quantize.restype = ctypes.c_int
    lib.fp4root_quantize_noalloc.argtypes = [vp, i64, i64, i64, i64, i64, ctypes.c_int, u32, f32, u64, i32,
                                             vp, vp, vp, vp, vp, vp]
    lib.fp4root_quantize_noalloc.restype = ctypes.c_int
    lib.fp4root_ns_step.argtypes = [vp, i64, i64, i64, i64, f32, f32, f32, u32, u64, i32,
                                    ctypes.POINTER(NsTrace), vp, sz, vp]
    lib.fp4root_ns_step.restype = ctypes.c_int
    lib.fp4root_orthogonalize.argtypes = [ctypes.POINTER(Matrix), i64, ctypes.POINTER(NsConfig), vp, sz, vp]
    lib.fp4root_orthogonalize.restype = ctypes.c_int
    lib.fp4root_momentum_workspace.argtypes = [i64, i64, i64]
    lib.fp4root_momentum_workspace.restype = sz
    lib.fp4root_momentum_update.argtypes = [vp, vp, i64, i64, i64, vp, vp, vp, f32, u32, u64, i32, vp, sz, vp]
    lib.fp4root_momentum_update.restype = ctypes.c_int
    lib.fp4root_qadamw_workspace.argtypes = [i64]
    lib.fp4root_qadamw_workspace.restype = sz
    lib.fp4root_qadamw_update.argtypes = [vp, vp, vp, i64, vp, vp, vp, vp, vp, vp, f32, f32, f32, f32, f32,
                                          u32, u64, i32, vp, sz, vp]
    lib.fp4root_qadamw_update.restype = ctypes.c_int
    lib.fp4root_apply_update.argtypes = [vp, vp, i64, f32, f32, f32, vp]
    lib.fp4root_apply_update.restype = ctypes.c_int
    lib.fp4root_root_step_workspace.argtypes = [ctypes.POINTER(Param), i64, ctypes.POINTER(NsConfig)]
    lib.fp4root_root_step_workspace.restype = sz
    lib.fp4root_root_step.argtypes = [ctypes.POINTER(Param), i64, ctypes.POINTER(RootConfig),
                                      ctypes.POINTER(NsConfig), vp, sz, vp]
    lib.fp4root_root_step.restype = ctypes.c_int
    lib.fp4root_grad_list_size.argtypes = [ctypes.POINTER(Tensor), i64]
    lib.fp4root_grad_list_size.restype = sz
    lib.fp4root_grad_list_init.argtypes = [ctypes.POINTER(GradList), ctypes.POINTER(Tensor), i64, vp, sz, vp]
    lib.fp4root_grad_list_init.restype = ctypes.c_int
    lib.fp4root_grad_norm.argtypes = [ctypes.POINTER(GradList), ctypes.c_int, f64, f64, vp, vp, vp, vp]
    lib.fp4root_grad_norm.restype = ctypes.c_int
    lib.fp4root_clip_coef.argtypes = [vp, ctypes.c_int, f64, f64, vp, vp]
    lib.fp4root_clip_coef.restype = ctypes.c_int
    lib.fp4root_clip_grads.argtypes = [ctypes.POINTER(GradList), vp, vp]
    lib.fp4root_clip_grads.restype = ctypes.c_int
    lib.fp4root_momentum_update_scaled.argtypes = [vp, vp, i64, i64, i64, vp, vp, vp, f32, u32, u64, i32, vp, vp, sz,
                                                   vp]
    lib.fp4root_momentum_update_scaled.restype = ctypes.c_int
    lib.fp4root_qadamw_update_scaled.argtypes = [vp, vp, vp, i64, vp, vp, vp, vp, vp, vp, f32, f32, f32, f32, f32,
                                                 u32, u64, i32, vp, vp, sz, vp]
    lib.fp4root_qadamw_update_scaled.restype = ctypes.c_int
    lib.fp4root_root_step_scaled.argtypes = [ctypes.POINTER(Param), i64, ctypes.POINTER(RootConfig),
                                             ctypes.POINTER(NsConfig), vp, vp, sz, vp]
    lib.fp4root_root_step_scaled.restype = ctypes.c_int
    lib.fp4root_rmsnorm_quantize.argtypes = [ctypes.POINTER(RmsNorm), vp]
    lib.fp4root_rmsnorm_quantize.restype = ctypes.c_int
    lib.fp4root_rmsnorm_backward_workspace.argtypes = [i64, i64]
    lib.fp4root_rmsnorm_backward_workspace.restype = sz
    lib.fp4root_rmsnorm_backward.argtypes = [vp, i64, vp, i64, vp, i64, vp, vp, vp, i64, vp, i64, i64, ctypes.c_int,
                                             ctypes.c_int, vp, sz, vp]
    lib.fp4root_rmsnorm_backward.restype = ctypes.c_int
    lib.fp4root_default_coeffs.argtypes = [i64, i64, i32, ctypes.POINTER(ctypes.c_float)]
    lib.fp4root_default_coeffs.restype = ctypes.c_int
    lib.fp4root_device_status.argtypes = [vp, vp]
    lib.fp4root_device_status.restype = ctypes.c_int
    lib.fp4root_status_string.argtypes = [ctypes.c_int]
    lib.fp4root_status_string.restype = ctypes.c_char_p
    lib.fp4root_version.argtypes = []
    lib.fp4root_version.restype = ctypes.c_int
    lib.fp4root_set_product_tiling.argtypes = [ctypes.c_int]
    lib.fp4root_set_product_tiling.restype = ctypes.c_int
    lib.fp4root_timer_enable.argtypes = [ctypes.c_int]
    lib.fp4root_timer_enable.restype = ctypes.c_int
    lib.fp4root_timer_read.argtypes = [ctypes.c_int, ctypes.POINTER(ctypes.c_double),
                                       ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_double)]
    lib.fp4root_timer_read.restype = ctypes.c_int
    lib.fp4root_timer_reset.argtypes = []
    lib.fp4root_timer_reset.restype = ctypes.c_int
    _lib = lib
    return lib


def header_symbols(path: str = HEADER) -> list[str]:
    """Names of the functions include/fp4root.h declares."""
    text = open(path).read()
    return sorted(set(re.findall(r"^\s*(?:const char\*|int|size_t)\s+(fp4root_\w+)\s*\(", text, re.M)))


def status_string(code: int) -> str:
    return load().fp4root_status_string(code).decode()


def _check(code: int, where: str):
    if code != OK:
        raise Fp4RootError(code, where)


def _stream(stream=None):
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else None


def _need_gpu_f32(x: torch.Tensor, name: str):
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if x.dtype != torch.float32:
        raise TypeError(f"{name} must be float32")


def _grad_scale(t, device):
    if t is None:
        return None
    _need_gpu_f32(t, "grad_scale")
    if t.numel() != 1 or t.device != device:
        raise ValueError("grad_scale must be one element on the gradients' GPU")
    return _ptr(t)


def workspace(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def fp4root_version() -> int:
    return load().fp4root_version()


def fp4root_set_product_tiling(mode: int) -> int:
    """0: tile form chosen per launch, 1: narrow (32 x 32 per wave), 2: wide (64 x 64);
    returns the previous mode.  Outputs are the same bits in every mode."""
    code = load().fp4root_set_product_tiling(int(mode))
    if code < 0:
        raise Fp4RootError(code, "fp4root_set_product_tiling")
    return code


def fp4root_timer_enable(on: bool = True):
    _check(load().fp4root_timer_enable(1 if on else 0), "fp4root_timer_enable")


def fp4root_timer_read(kernel: int = -1):
    """(total kernel ms, launches, algorithmic FLOP) of the recorded product launches."""
    ms, n, fl = ctypes.c_double(), ctypes.c_int64(), ctypes.c_double()
    _check(load().fp4root_timer_read(kernel, ctypes.byref(ms), ctypes.byref(n), ctypes.byref(fl)),
           "fp4root_timer_read")
    return ms.value, n.value, fl.value


def fp4root_timer_reset():
    _check(load().fp4root_timer_reset(), "fp4root_timer_reset")


def fp4root_default_coeffs(rows: int, cols: int, steps: int = 5):
    buf = (ctypes.c_float * (3 * steps))()
    _check(load().fp4root_default_coeffs(rows, cols, steps, buf), "fp4root_default_coeffs")
    return [(buf[3 * k], buf[3 * k + 1], buf[3 * k + 2]) for k in range(steps)]


def fp4root_device_status(ws: torch.Tensor, stream=None) -> int:
    return load().fp4root_device_status(_ptr(ws), _stream(stream))


def fp4root_quantize(x: torch.Tensor, axis: int = 1, flags: int = F_HADAMARD | F_ADAPTIVE46,
                     clip_quantile: float = 0.99, seed: int = 0, step: int = 0, ws=None, stream=None):
    """NVFP4-quantise a matrix or a batch (B, rows, cols) of float32 matrices.

    Returns (codes, scales, tensor_scale, clip_threshold, ws); codes hold two
    4-bit codes per byte.  See fp4root_quantize in include/fp4root.h.
    """
    _need_gpu_f32(x, "x")
    lib = load()
    xb = x if x.dim() == 3 else x.unsqueeze(0)
    if xb.stride(-1) != 1:
        raise ValueError("x rows must be contiguous")
    B, R, C = xb.shape
    ld = xb.stride(1)
    bstride = xb.stride(0) if B > 1 else R * ld
    dev = x.device
    if axis == 1:
        codes = torch.empty((B, R, C // 2), dtype=torch.uint8, device=dev)
        scales = torch.empty((B, R, C // 16), dtype=torch.uint8, device=dev)
    else:
        codes = torch.empty((B, C, R // 2), dtype=torch.uint8, device=dev)
        scales = torch.empty((B, C, R // 16), dtype=torch.uint8, device=dev)
    sg = torch.empty(B, dtype=torch.float32, device=dev)
    tau = torch.empty(B, dtype=torch.float32, device=dev)
    need = lib.fp4root_quantize_workspace(B, R, C, flags)
    if ws is None or ws.numel() < need:
        ws = workspace(need, dev)
    _check(lib.fp4root_quantize(_ptr(xb), B, R, C, ld, bstride, axis, flags, clip_quantile, seed,
                                step, _ptr(codes), _ptr(scales), _ptr(sg), _ptr(tau), _ptr(ws),
                                ws.numel(), _stream(stream)), "fp4root_quantize")
    if x.dim() == 2:
        codes, scales = codes[0], scales[0]
    return codes, scales, sg, tau, ws


def fp4root_quantize_noalloc(x: torch.Tensor, out, axis: int = 1, flags: int = F_HADAMARD | F_ADAPTIVE46,
                             clip_quantile: float = 0.99, seed: int = 0, step: int = 0, stream=None):
    """fp4root_quantize into caller-owned outputs without a workspace (the library's
    fixed scratch; at most 256 matrices with clipping, 1166 without).  out = (codes, scales, tensor_scale,
    clip_threshold or None, status or None), shaped as fp4root_quantize returns them
    (batch first); status is an int32 device tensor of one element."""
    _need_gpu_f32(x, "x")
    codes, scales, sg, tau, status = out
    xb = x if x.dim() == 3 else x.unsqueeze(0)
    if xb.stride(-1) != 1:
        raise ValueError("x rows must be contiguous")
    B, R, C = xb.shape
    ld = xb.stride(1)
    bstride = xb.stride(0) if B > 1 else R * ld
    _check(load().fp4root_quantize_noalloc(_ptr(xb), B, R, C, ld, bstride, axis, flags, clip_quantile, seed, step,
                                           _ptr(codes), _ptr(scales), _ptr(sg),
                                           _ptr(tau) if tau is not None else None,
                                           _ptr(status) if status is not None else None, _stream(stream)),
           "fp4root_quantize_noalloc")


def fp4root_ns_step(x: torch.Tensor, a: float, b: float, c: float,
                    flags: int = F_HADAMARD | F_ADAPTIVE46, seed: int = 0, step: int = 0,
                    trace: bool = False, ws=None, stream=None):
    """One NS step in place on x (m, n) or (B, m, n).  With trace=True returns a dict of
    the step's intermediates (qX, qXt, A, qA, B, qB), else None."""
    _need_gpu_f32(x, "x")
    if not x.is_contiguous():
        raise ValueError("x must be contiguous")
    lib = load()
    xb = x if x.dim() == 3 else x.unsqueeze(0)
    B, m, n = xb.shape
    need = lib.fp4root_ns_step_workspace(B, m, n, flags)
    if ws is None or ws.numel() < need:
        ws = workspace(need, x.device)
    tr = None
    out = None
    if trace:
        dev = x.device
        u8 = dict(dtype=torch.uint8, device=dev)
        f32 = dict(dtype=torch.float32, device=dev)
        out = {
            "qx_codes": torch.empty((B, m, n // 2), **u8), "qx_scales": torch.empty((B, m, n // 16), **u8),
            "qx_sg": torch.empty(B, **f32),
            "qxt_codes": torch.empty((B, n, m // 2), **u8), "qxt_scales": torch.empty((B, n, m // 16), **u8),
            "qxt_sg": torch.empty(B, **f32),
            "A": torch.empty((B, m, m), **f32),
            "qa_codes": torch.empty((B, m, m // 2), **u8), "qa_scales": torch.empty((B, m, m // 16), **u8),
            "qa_sg": torch.empty(B, **f32),
            "B": torch.empty((B, m, m), **f32),
            "qb_codes": torch.empty((B, m, m // 2), **u8), "qb_scales": torch.empty((B, m, m // 16), **u8),
            "qb_sg": torch.empty(B, **f32),
        }
        tr = NsTrace(**{k: v.data_ptr() for k, v in out.items()})
    _check(lib.fp4root_ns_step(_ptr(xb), B, m, n, m * n, a, b, c, flags, seed, step,
                               ctypes.byref(tr) if tr is not None else None, _ptr(ws), ws.numel(),
                               _stream(stream)), "fp4root_ns_step")
    return out


class MomentumState:
    """NVFP4 first-moment state of a batch of rows x cols matrices (device tensors):
    codes (B, rows, cols/2), scales (B, rows, cols/16), tensor_scale (B,)."""

    def __init__(self, batch: int, rows: int, cols: int, device="cuda"):
        self.codes = torch.zeros((batch, rows, cols // 2), dtype=torch.uint8, device=device)
        self.scales = torch.zeros((batch, rows, cols // 16), dtype=torch.uint8, device=device)
        self.tensor_scale = torch.zeros(batch, dtype=torch.float32, device=device)
        self.ws = workspace(load().fp4root_momentum_workspace(batch, rows, cols), device)


def fp4root_momentum_update(g: torch.Tensor, state: MomentumState, beta: float, step: int,
                            flags: int = F_HADAMARD | F_ADAPTIVE46 | F_STOCHASTIC, seed: int = 0,
                            m: torch.Tensor = None, stream=None, grad_scale: torch.Tensor = None) -> torch.Tensor:
    """One first-moment step: returns m_t (FP32, shape of g) and re-encodes `state`.
    g: (rows, cols) or (B, rows, cols) contiguous float32; grad_scale: a float32 GPU
    tensor of one element that multiplies g (GradClipper.coef).  See include/fp4root.h."""
    _need_gpu_f32(g, "g")
    if not g.is_contiguous():
        raise ValueError("g must be contiguous")
    gb = g if g.dim() == 3 else g.unsqueeze(0)
    B, R, C = gb.shape
    if tuple(state.codes.shape) != (B, R, C // 2):
        raise ValueError("state shape does not match g")
    if m is None:
        m = torch.empty_like(g)
    _need_gpu_f32(m, "m")
    if m.shape != g.shape or not m.is_contiguous():
        raise ValueError("m must be a contiguous tensor of g's shape")
    _check(load().fp4root_momentum_update_scaled(
        _ptr(gb), _ptr(m), B, R, C, _ptr(state.codes), _ptr(state.scales), _ptr(state.tensor_scale), beta, flags, seed,
        step, _grad_scale(grad_scale, g.device), _ptr(state.ws), state.ws.numel(), _stream(stream)),
        "fp4root_momentum_update")
    return m


def fp4root_apply_update(w: torch.Tensor, o: torch.Tensor, lr: float, wd: float, scale: float, stream=None):
    """W <- bf16(fl32(fl32(W c1) - fl32(c2 O))) in place on a contiguous bfloat16 tensor w."""
    if w.dtype != torch.bfloat16 or not w.is_cuda or not w.is_contiguous():
        raise TypeError("w must be a contiguous bfloat16 GPU tensor")
    _need_gpu_f32(o, "o")
    if o.shape != w.shape or not o.is_contiguous():
        raise ValueError("o must be a contiguous float32 tensor of w's shape")
    _check(load().fp4root_apply_update(_ptr(w), _ptr(o), w.numel(), lr, wd, scale, _stream(stream)),
           "fp4root_apply_update")


class QAdamWState:
    """Both quantized AdamW moments of a flat parameter of n elements (device tensors)."""

    def __init__(self, n: int, device="cuda", keep_m: bool = False):
        if n <= 0 or n % 256:
            raise ValueError("n must be a positive multiple of 256")
        self.n = n
        # this step's binary32 first moment, written only when kept (diagnostics)
        self.m = torch.empty(n, dtype=torch.float32, device=device) if keep_m else None
        self.m_codes = torch.zeros(n // 2, dtype=torch.uint8, device=device)
        self.m_scales = torch.zeros(n // 16, dtype=torch.uint8, device=device)
        self.m_tensor_scale = torch.zeros(1, dtype=torch.float32, device=device)
        self.v_codes = torch.zeros(n // 2, dtype=torch.uint8, device=device)
        self.v_scales = torch.zeros(n // 16, dtype=torch.int16, device=device)
        self.v_means = torch.zeros(n // 256, dtype=torch.int16, device=device)
        self.ws = workspace(load().fp4root_qadamw_workspace(n), device)


def fp4root_qadamw_update(w: torch.Tensor, g: torch.Tensor, state: QAdamWState, step: int, lr: float,
                          wd: float = 0.1, beta1: float = 0.9, beta2: float = 0.95, eps: float = 1e-8,
                          flags: int = F_HADAMARD | F_ADAPTIVE46 | F_STOCHASTIC, seed: int = 0, stream=None,
                          grad_scale: torch.Tensor = None):
    """One quantized-state AdamW step on a flat contiguous bfloat16 parameter w with FP32 gradient g
    (times grad_scale, a float32 GPU tensor of one element, if given)."""
    if w.dtype != torch.bfloat16 or not w.is_cuda or not w.is_contiguous():
        raise TypeError("w must be a contiguous bfloat16 GPU tensor")
    _need_gpu_f32(g, "g")
    if g.numel() != w.numel() or not g.is_contiguous() or w.numel() != state.n:
        raise ValueError("g and state must match w")
    _check(load().fp4root_qadamw_update_scaled(
        _ptr(w), _ptr(g), _ptr(state.m), state.n, _ptr(state.m_codes), _ptr(state.m_scales),
        _ptr(state.m_tensor_scale), _ptr(state.v_codes), _ptr(state.v_scales), _ptr(state.v_means),
        lr, wd, beta1, beta2, eps, flags, seed, step, _grad_scale(grad_scale, w.device), _ptr(state.ws),
        state.ws.numel(), _stream(stream)), "fp4root_qadamw_update")


class RootStep:
    """Reusable fp4root_root_step over a fixed list of (BF16 weight, FP32 gradient) pairs.

    Holds the descriptors, each parameter's first-moment state and FP32 scratch,
    the configurations and the workspace; each call is one C call.  With max_norm every call
    first takes the gradients' global norm (self.clipper, a GradClipper) and the step reads
    them times its clipping coefficient; a norm over more tensors than these is taken by a
    GradClipper of the caller's, whose coef goes into the call as grad_scale.
    """

    def __init__(self, weights, grads, lr: float, wd: float = 0.1, beta: float = 0.9, steps: int = 5,
                 coeffs=None, ns_flags: int = F_DEFAULT, momentum_flags: int = F_HADAMARD | F_ADAPTIVE46 | F_STOCHASTIC,
                 clip_quantile: float = 0.99, eps: float = 1e-7, seed: int = 0, momentum_seed: int = 0,
                 scales=None, max_norm: float = None):
        lib = load()
        self.weights, self.grads = list(weights), list(grads)
        n = len(self.weights)
        self.scratch, self.states = [], []
        self.params = (Param * max(n, 1))()
        for i, (w, g) in enumerate(zip(self.weights, self.grads)):
            if w.dtype != torch.bfloat16 or not w.is_cuda or not w.is_contiguous() or w.dim() != 2:
                raise TypeError(f"weights[{i}] must be a contiguous 2-D bfloat16 GPU tensor")
            _need_gpu_f32(g, f"grads[{i}]")
            if g.shape != w.shape or not g.is_contiguous():
                raise ValueError(f"grads[{i}] must be contiguous with the weight's shape")
            r, c = w.shape
            m = torch.empty_like(g)
            st = MomentumState(1, r, c, device=w.device)
            self.scratch.append(m)
            self.states.append(st)
            sc = scales[i] if scales is not None else 0.0   # 0: the library's default scale
            self.params[i] = Param(w.data_ptr(), g.data_ptr(), m.data_ptr(), st.codes.data_ptr(),
                                   st.scales.data_ptr(), st.tensor_scale.data_ptr(), r, c, sc)
        self.count = n
        if coeffs is not None:
            flat = [float(v) for row in coeffs for v in row]
            if len(flat) != 3 * steps:
                raise ValueError("coeffs must hold steps rows of (a, b, c)")
            self._coeffs = (ctypes.c_float * len(flat))(*flat)
            cptr = ctypes.cast(self._coeffs, ctypes.POINTER(ctypes.c_float))
        else:
            self._coeffs, cptr = None, None
        self.ns = NsConfig(steps, cptr, ns_flags, clip_quantile, eps, seed)
        self.cfg = RootConfig(lr, wd, beta, momentum_flags, momentum_seed, 0)
        need = lib.fp4root_root_step_workspace(self.params, n, ctypes.byref(self.ns))
        if need == 0:
            raise ValueError("invalid parameters or configuration")
        self.ws = workspace(need, self.weights[0].device if n else torch.device("cuda"))
        self.clipper = GradClipper(self.grads, max_norm, measure_only=True) if max_norm is not None and n else None

    def __call__(self, step: int, stream=None, grad_scale: torch.Tensor = None):
        self.cfg.step = step
        if self.clipper is not None:
            if grad_scale is not None:
                raise ValueError("max_norm and grad_scale exclude each other")
            self.clipper.norm(stream)
            grad_scale = self.clipper.coef
        scale = _grad_scale(grad_scale, self.ws.device)
        _check(load().fp4root_root_step_scaled(self.params, self.count, ctypes.byref(self.cfg), ctypes.byref(self.ns),
                                               scale, _ptr(self.ws), self.ws.numel(), _stream(stream)),
               "fp4root_root_step")

    def status(self, stream=None) -> int:
        return fp4root_device_status(self.ws, stream)


def _launch_stream(device, stream) -> int:
    """The raw stream of a call on tensors of `device`: the given one, or the current one there."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(device.index)
    if stream.device != device:
        raise ValueError("the stream belongs to another GPU than the tensors")
    return stream.cuda_stream


def _call(fn, device, *args) -> int:
    """fn(*args) with `device` current: kernels are launched on the current GPU's code."""
    if device.index == torch._C._cuda_getDevice():
        return fn(*args)
    with torch.cuda.device(device):
        return fn(*args)


def _as_rows(t: torch.Tensor, name: str):
    """(rows, cols, row stride) under which a kernel walks t in the order of its memory."""
    if t.numel() == 0:
        return 0, 0, 0
    if t.is_contiguous():
        return 1, t.numel(), t.numel()
    order = sorted((i for i in range(t.dim()) if t.shape[i] > 1), key=lambda i: (t.stride(i), t.shape[i]))
    sizes = [(t.shape[i], t.stride(i)) for i in order]
    if sizes[0][1] != 1:
        sizes.insert(0, (1, 1))
    cols, k = sizes[0][0], 1
    while k < len(sizes) and sizes[k][1] == cols:      # the innermost run of memory
        cols *= sizes[k][0]
        k += 1
    rows, ld = 1, sizes[k][1] if k < len(sizes) else cols
    while k < len(sizes) and sizes[k][1] == rows * ld:
        rows *= sizes[k][0]
        k += 1
    if k < len(sizes) or (rows > 1 and ld < cols):
        raise ValueError(f"{name} must be rows of one stride (contiguous, a slice of columns, or a transpose of these)")
    return rows, cols, ld


class GradClipper:
    """The global norm of a fixed list of gradient tensors (float32, bfloat16 or float16, mixed
    as they come) and the clipping by it; see fp4root_grad_norm and fp4root_clip_grads in
    include/fp4root.h.  Holds the list, its device memory and the results:

      total       float64 [1]: the sum of squares (norm_type 2) or largest magnitude (inf)
      norms       float32 [len(grads)]: each tensor's norm
      total_norm  float32 scalar, coef float32 scalar: min(1, max_norm / (total_norm + eps))

    `norm()` computes these; a call computes them and multiplies every gradient by coef, into
    `outputs` (tensors of the gradients' shapes and any of the types, or None: in place).  Ranks
    that hold shards run `norm()`, all-reduce `total` (sum, or maximum for inf), then `recoef()`
    and `scale()`; status() goes on to speak of the rank's own shard.  With measure_only there is
    nothing to scale, and a tensor may be listed twice
    (it counts twice).  RootStep, fp4root_qadamw_update and fp4root_momentum_update take `coef` as
    grad_scale and then need no scaled gradients.  Each may be captured into a HIP graph, and
    used on any stream once the object is made (it waits for its own set-up); calls of one
    GradClipper on two streams at once race.  It reads the tensors it was made with: a gradient that
    a later step puts into a new tensor (a `.grad` set to None in between, a dgain that
    fp4root_rmsnorm_backward allocates) is not seen, so give such producers their buffer.  The
    gradients' memory must stay where it is, and the object alive, until its calls have run.
    """

    def __init__(self, grads, max_norm: float, outputs=None, norm_type=2, eps: float = 1e-6,
                 measure_only: bool = False):
        self._make(grads, max_norm, outputs, norm_type, eps, measure_only)
        if self.count:
            torch.cuda.current_stream(self.device).synchronize()

    def _make(self, grads, max_norm, outputs, norm_type, eps, measure_only):
        lib = load()
        self.grads = list(grads)
        self.outputs = list(outputs) if outputs is not None else self.grads
        if len(self.outputs) != len(self.grads) or (measure_only and outputs is not None):
            raise ValueError("outputs must match grads")
        if norm_type not in (2, float("inf")):
            raise ValueError("norm_type must be 2 or inf")
        if not max_norm > 0 or not 0 <= eps < float("inf"):
            raise ValueError("max_norm must be positive and eps non-negative")
        self.kind = NORM_L2 if norm_type == 2 else NORM_MAX
        self.max_norm, self.eps = float(max_norm), float(eps)
        n = self.count = len(self.grads)
        tensors = (Tensor * max(n, 1))()
        for i, (g, o) in enumerate(zip(self.grads, self.outputs)):
            for name, t in ((f"grads[{i}]", g), (f"outputs[{i}]", o)):
                if not isinstance(t, torch.Tensor) or not t.is_cuda or t.device != self.grads[0].device:
                    raise TypeError(f"{name} must be a tensor on the first gradient's GPU")
                if t.dtype not in _TYPES:
                    raise TypeError(f"{name} must be float32, bfloat16 or float16")
            rows, cols, ld = _as_rows(g, f"grads[{i}]")
            ld_out = ld
            if o is not g:
                rows, cols, ld, ld_out = _rows_of_both(g, o, rows, cols, ld, i)
            tensors[i] = Tensor(g.data_ptr(), None if measure_only else o.data_ptr(), rows, cols, ld, ld_out,
                                _TYPES[g.dtype], _TYPES[o.dtype])
        self.device = self.grads[0].device if n else torch.device("cuda", torch.cuda.current_device())
        need = lib.fp4root_grad_list_size(tensors, n)
        if need == 0:
            raise ValueError("invalid gradients")
        self.ws = workspace(need, self.device)
        self.total = torch.zeros(1, dtype=torch.float64, device=self.device)
        self.norms = torch.zeros(n, dtype=torch.float32, device=self.device)
        self.result = torch.zeros(2, dtype=torch.float32, device=self.device)
        self.total_norm, self.coef = self.result[0], self.result[1]
        self.list = GradList()
        _check(_call(lib.fp4root_grad_list_init, self.device, ctypes.byref(self.list), tensors, n, _ptr(self.ws),
                     self.ws.numel(), _launch_stream(self.device, None)), "fp4root_grad_list_init")
        self._list = ctypes.byref(self.list)
        self._norm_args = (self._list, self.kind, self.max_norm, self.eps, _ptr(self.total),
                           _ptr(self.norms) if n else None, _ptr(self.result))

    def norm(self, stream=None) -> torch.Tensor:
        """The norm (self.total_norm), and with it total, norms and coef."""
        _check(_call(_lib.fp4root_grad_norm, self.device, *self._norm_args, _launch_stream(self.device, stream)),
               "fp4root_grad_norm")
        return self.total_norm

    def recoef(self, stream=None) -> torch.Tensor:
        """total_norm and coef again, from `total` (after an all-reduce)."""
        _check(_call(_lib.fp4root_clip_coef, self.device, _ptr(self.total), self.kind, self.max_norm, self.eps,
                     _ptr(self.result), _launch_stream(self.device, stream)), "fp4root_clip_coef")
        return self.total_norm

    def scale(self, stream=None):
        """Every gradient times coef, into the outputs, which it returns."""
        _check(_call(_lib.fp4root_clip_grads, self.device, self._list, _ptr(self.coef),
                     _launch_stream(self.device, stream)), "fp4root_clip_grads")
        return self.outputs

    def __call__(self, stream=None):
        self.norm(stream)
        return self.scale(stream)

    def status(self, stream=None) -> int:
        """FP4ROOT_ERR_NONFINITE where the last norm met a NaN or an infinity, else 0 (waits)."""
        return _call(_lib.fp4root_device_status, self.device, _ptr(self.ws), _launch_stream(self.device, stream))


def _rows_of_both(g, o, rows, cols, ld, i):
    """(rows, cols, row stride, output's row stride) under which both are walked alike."""
    if o.shape != g.shape:
        raise ValueError(f"outputs[{i}] must have the gradient's shape")
    ri, ci, ld_out = _as_rows(o, f"outputs[{i}]")
    dims = [d for d in range(g.dim()) if g.shape[d] > 1]
    if sorted(dims, key=lambda d: g.stride(d)) != sorted(dims, key=lambda d: o.stride(d)):
        raise ValueError(f"outputs[{i}] must have its dimensions in memory in the gradient's order")
    if (ri, ci) != (rows, cols):       # a contiguous one beside one of rows is taken as those rows
        if ri == 1 and rows * cols == ci:
            ld_out = cols
        elif rows == 1 and ri * ci == cols:
            rows, cols, ld = ri, ci, ci
        else:
            raise ValueError(f"outputs[{i}] must be laid out as the gradient, or contiguous")
    return rows, cols, ld, ld_out


def fp4root_clip_grads(grads, max_norm: float, outputs=None, norm_type=2, eps: float = 1e-6, stream=None):
    """Clip a list of gradient tensors by their global norm, in place or into `outputs`; returns
    the norm before clipping (a float32 GPU scalar).  A program that clips the same buffers step
    after step keeps a GradClipper instead."""
    grads = list(grads)
    if stream is not None:        # allocated where it is used
        if grads:
            _launch_stream(grads[0].device, stream)
        with torch.cuda.stream(stream):
            return fp4root_clip_grads(grads, max_norm, outputs, norm_type, eps)
    c = GradClipper.__new__(GradClipper)
    c._make(grads, max_norm, outputs, norm_type, eps, False)
    c()
    return c.total_norm


class RmsNormOutput(NamedTuple):
    """codes: uint8 E4M3FN codes of the input's shape; scales: float32, or uint8 exponents
    (E8M0); rstd: float32 per row; h: the stream after the residual's addition (x itself
    without a residual); y: the unquantized output if wanted."""
    codes: Optional[torch.Tensor]
    scales: Optional[torch.Tensor]
    rstd: torch.Tensor
    h: torch.Tensor
    y: Optional[torch.Tensor]


class _Unadded(RmsNormOutput):
    """The result of a call without a residual: its h is the caller's x and no output, unless the
    caller makes another tensor h."""
    __slots__ = ()

    def _replace(self, **fields):
        got = super()._replace(**fields)
        return RmsNormOutput(*got) if "h" in fields else got


def _matrix(t: torch.Tensor, name: str, like: torch.Tensor = None):
    """(rows, row stride) of a tensor whose last dimension is contiguous and whose others are
    rows of one stride; checked against `like`, an accepted one, for type, shape and GPU."""
    if like is not None and (not isinstance(t, torch.Tensor) or t.dtype is not like.dtype or t.shape != like.shape or
                             t.device != like.device):
        raise TypeError(f"{name} must have x's type, shape and GPU")
    cols = t.shape[-1]
    if t.is_contiguous():
        return (t.numel() // cols if cols else 0), cols
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name} rows must be contiguous")
    lead = [(t.shape[i], t.stride(i)) for i in range(t.dim() - 1) if t.shape[i] > 1]
    rows, ld = 1, t.shape[-1]
    for k, (n, s) in enumerate(reversed(lead)):
        if k == 0:
            ld = s
        elif s != rows * ld:
            raise ValueError(f"{name} must be rows of one stride")
        rows *= n
    if rows > 1 and ld < t.shape[-1]:
        raise ValueError(f"{name} rows must not overlap")
    return (0 if t.numel() == 0 else rows), ld


def _gain_type(gain, x):
    if gain is None:
        return FLOAT32
    code = _GAIN_TYPES.get(gain.dtype) if isinstance(gain, torch.Tensor) and gain.device == x.device else None
    if code is None:
        raise TypeError("gain must be a float32 or bfloat16 tensor on x's GPU")
    if gain.shape != x.shape[-1:] or not gain.is_contiguous():
        raise ValueError("gain must be a contiguous vector of x's columns")
    return code


def _need_stream(x, name: str) -> int:
    """The type of a matrix that a norm reads, checked."""
    if _lib is None:
        load()
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    code = _TYPES.get(x.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32, bfloat16 or float16")
    if x.dim() < 1:
        raise ValueError(f"{name} must have a dimension of columns")
    return code


def fp4root_rmsnorm_quantize(x: torch.Tensor, gain: torch.Tensor = None, residual: torch.Tensor = None,
                             eps: float = 1e-6, group: int = 0, e8m0: bool = False, quantize: bool = True,
                             want_y: bool = False, out: RmsNormOutput = None, status: torch.Tensor = None,
                             stream=None) -> RmsNormOutput:
    """h = x + residual, then its root-mean-square norm times gain, in E4M3 with a scale per row
    (group 0) or per group of 32, 64 or 128 columns.  x: (..., cols), float32, bfloat16 or
    float16, rows of one stride; out: an earlier call's result, whose tensors are written again
    (out._replace(h=...) with the residual or x itself: in place), but for the h of a call without a
    residual, which is that call's x and is replaced; status: an int32 GPU tensor of one element.
    See fp4root_rmsnorm_quantize in include/fp4root.h."""
    if stream is not None:        # allocated where it is used
        _launch_stream(x.device, stream)
        with torch.cuda.stream(stream):
            return fp4root_rmsnorm_quantize(x, gain, residual, eps, group, e8m0, quantize, want_y, out, status)
    type_ = _need_stream(x, "x")
    shape, dev, packed = x.shape, x.device, x.is_contiguous()
    lead, cols = shape[:-1], shape[-1]
    rows, ld_x = (x.numel() // cols, cols) if packed and cols else _matrix(x, "x")
    gain_type = ld_r = ld_h = ld_y = 0
    gain_p = r_p = h_p = y_p = codes_p = scales_p = rstd_p = status_p = None
    if gain is not None:
        gain_type, gain_p = _gain_type(gain, x), gain.data_ptr()
    if residual is not None:
        ld_r, r_p = _matrix(residual, "residual", x)[1], residual.data_ptr()
    if out is None:
        # empty_like keeps a stride, and is the cheaper call
        codes = scales = y = None
        if quantize:
            codes = torch.empty_like(x, dtype=torch.uint8) if packed else x.new_empty(shape, dtype=torch.uint8)
            scales = x.new_empty((*lead, -(-cols // group)) if group > 0 else lead,
                                 dtype=torch.uint8 if e8m0 else torch.float32)
            codes_p, scales_p = codes.data_ptr(), scales.data_ptr()
        rstd = torch.empty_like(scales) if quantize and group == 0 and not e8m0 else \
            x.new_empty(lead, dtype=torch.float32)
        rstd_p, h = rstd.data_ptr(), x
        if residual is not None:
            h, ld_h = torch.empty_like(x) if packed else x.new_empty(shape), cols
            h_p = h.data_ptr()
        if want_y:
            y, ld_y = x.new_empty(shape), cols
            y_p = y.data_ptr()
        out = (RmsNormOutput if residual is not None else _Unadded)(codes, scales, rstd, h, y)
    else:
        codes, scales, rstd, h, y = out
        for name, t, dtype, want in (("codes", codes, torch.uint8, shape),
                                     ("scales", scales, torch.uint8 if e8m0 else torch.float32,
                                      (*lead, -(-cols // group)) if group > 0 else lead),
                                     ("rstd", rstd, torch.float32, lead)):
            if t is not None and (t.dtype != dtype or tuple(t.shape) != tuple(want) or not t.is_contiguous() or
                                  t.device != dev):
                raise ValueError(f"out.{name} must be a contiguous {dtype} tensor of shape {tuple(want)} on x's GPU")
        if residual is None:
            out = _Unadded(codes, scales, rstd, x, y)      # the stream is x: nothing to write
        elif type(out) is _Unadded:
            h = torch.empty_like(x) if packed else x.new_empty(shape)
            out = RmsNormOutput(codes, scales, rstd, h, y)
        if residual is not None and h is not None:
            ld_h, h_p = _matrix(h, "out.h", x)[1], h.data_ptr()
        if y is not None:
            ld_y, y_p = _matrix(y, "out.y", x)[1], y.data_ptr()
        codes_p, scales_p, rstd_p = (t.data_ptr() if t is not None else None for t in (codes, scales, rstd))
    if status is not None:
        if status.dtype != torch.int32 or status.numel() != 1 or status.device != dev:
            raise ValueError("status must be one int32 element on x's GPU")
        status_p = status.data_ptr()
    a = RmsNorm(x.data_ptr(), r_p, gain_p, h_p, y_p, codes_p, scales_p, rstd_p, status_p, rows, cols, ld_x, ld_r,
                ld_h, ld_y, type_, gain_type, group, SCALE_E8M0 if e8m0 else SCALE_FP32, eps)
    _check(_call(_lib.fp4root_rmsnorm_quantize, dev, ctypes.byref(a), _launch_stream(dev, None)),
           "fp4root_rmsnorm_quantize")
    return out


def fp4root_rmsnorm_backward(dy: torch.Tensor, h: torch.Tensor, gain: Optional[torch.Tensor], rstd: torch.Tensor,
                             dh: torch.Tensor = None, dx: torch.Tensor = None, dgain: torch.Tensor = None,
                             want_dgain: bool = True, ws: torch.Tensor = None, stream=None):
    """(dx, dgain) of the norm of h under the gradient dy of its output and dh of h itself; dx in
    h's type is the gradient of x and of the residual alike, dgain is float32.  dx may be given
    (dy, h or dh itself: in place); see fp4root_rmsnorm_backward in include/fp4root.h."""
    if stream is not None:        # allocated where it is used
        _launch_stream(h.device, stream)
        with torch.cuda.stream(stream):
            return fp4root_rmsnorm_backward(dy, h, gain, rstd, dh, dx, dgain, want_dgain, ws)
    type_ = _need_stream(h, "h")
    rows, ld_h = _matrix(h, "h")
    ld_dy = _matrix(dy, "dy", h)[1]
    ld_dh = _matrix(dh, "dh", h)[1] if dh is not None else 0
    cols, dev = h.shape[-1], h.device
    gain_type = _gain_type(gain, h)
    _need_gpu_f32(rstd, "rstd")
    if rstd.numel() != rows or not rstd.is_contiguous() or rstd.device != dev:
        raise ValueError("rstd must hold one contiguous element per row on h's GPU")
    if dx is None:
        dx = torch.empty_like(h) if ld_h == cols and h.is_contiguous() else h.new_empty(h.shape)
        ld_dx = cols
    else:
        ld_dx = _matrix(dx, "dx", h)[1]
    if dgain is not None:
        _need_gpu_f32(dgain, "dgain")
        if dgain.numel() != cols or not dgain.is_contiguous() or dgain.device != dev:
            raise ValueError("dgain must hold one contiguous element per column on h's GPU")
    elif want_dgain:
        dgain = h.new_empty(cols, dtype=torch.float32)
    dgain_p = ws_p = None
    ws_bytes = 0
    if dgain is not None:
        if ws is None:
            ws = h.new_empty(_lib.fp4root_rmsnorm_backward_workspace(rows, cols), dtype=torch.uint8)
        elif ws.device != dev or not ws.is_contiguous():
            raise ValueError("ws must be contiguous on h's GPU")
        dgain_p, ws_p, ws_bytes = dgain.data_ptr(), ws.data_ptr(), ws.numel() * ws.element_size()
    _check(_call(_lib.fp4root_rmsnorm_backward, dev, dy.data_ptr(), ld_dy, h.data_ptr(), ld_h,
                 dh.data_ptr() if dh is not None else None, ld_dh, gain.data_ptr() if gain is not None else None,
                 rstd.data_ptr(), dx.data_ptr(), ld_dx, dgain_p, rows, cols, type_, gain_type, ws_p, ws_bytes,
                 _launch_stream(dev, None)), "fp4root_rmsnorm_backward")
    return dx, dgain


class Orthogonalizer:
    """Reusable call of fp4root_orthogonalize over a fixed list of matrices.

    Holds the descriptor array, the configuration and the workspace so that a
    timed loop makes exactly one C call per invocation.
    """

    def __init__(self, inputs, outputs=None, steps: int = 5, coeffs=None, flags: int = F_DEFAULT,
                 clip_quantile: float = 0.99, eps: float = 1e-7, seed: int = 0):
        lib = load()
        self.inputs = list(inputs)
        self.outputs = list(outputs) if outputs is not None else [torch.empty_like(t) for t in self.inputs]
        n = len(self.inputs)
        self.mats = (Matrix * max(n, 1))()
        for i, (a, o) in enumerate(zip(self.inputs, self.outputs)):
            _need_gpu_f32(a, f"inputs[{i}]")
            _need_gpu_f32(o, f"outputs[{i}]")
            if a.dim() != 2 or a.stride(1) != 1 or o.stride(1) != 1 or o.shape != a.shape:
                raise ValueError(f"matrix {i}: need 2-D row-contiguous input and output of equal shape")
            self.mats[i] = Matrix(a.data_ptr(), o.data_ptr(), a.shape[0], a.shape[1], a.stride(0), o.stride(0))
        self.count = n
        if coeffs is not None:
            flat = [float(v) for row in coeffs for v in row]
            if len(flat) != 3 * steps:
                raise ValueError("coeffs must hold steps rows of (a, b, c)")
            self._coeffs = (ctypes.c_float * len(flat))(*flat)
            cptr = ctypes.cast(self._coeffs, ctypes.POINTER(ctypes.c_float))
        else:
            self._coeffs = None
            cptr = None
        self.cfg = NsConfig(steps, cptr, flags, clip_quantile, eps, seed)
        need = lib.fp4root_orthogonalize_workspace(self.mats, n, ctypes.byref(self.cfg))
        if need == 0:
            raise ValueError("invalid matrices or configuration")
        dev = self.inputs[0].device if n else torch.device("cuda")
        self.ws = workspace(need, dev)

    def __call__(self, stream=None):
        _check(load().fp4root_orthogonalize(self.mats, self.count, ctypes.byref(self.cfg),
                                            _ptr(self.ws), self.ws.numel(), _stream(stream)),
               "fp4root_orthogonalize")
        return self.outputs

    def capture(self):
        """Record one call into a HIP graph (the library allocates nothing and clears
        its scalars with kernels, so the whole call can be captured); returns the graph,
        whose replay() repeats the call on the same buffers."""
        graph = torch.cuda.CUDAGraph()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            self()                       # warm call outside the capture
        torch.cuda.current_stream().wait_stream(side)
        with torch.cuda.graph(graph, stream=side):
            self()
        torch.cuda.synchronize()
        return graph

    def status(self, stream=None) -> int:
        return fp4root_device_status(self.ws, stream)


def fp4root_orthogonalize(inputs, outputs=None, steps: int = 5, coeffs=None, flags: int = F_DEFAULT,
                          clip_quantile: float = 0.99, eps: float = 1e-7, seed: int = 0, stream=None):
    """Orthogonalise a list of float32 GPU matrices; returns the outputs (new tensors unless given)."""
    return Orthogonalizer(inputs, outputs, steps, coeffs, flags, clip_quantile, eps, seed)(stream)
