"""Thin Python binding of include/lsh_qk.h: per-head norm with position rotation.

``lsh_qk_norm_rotate_fwd`` and ``lsh_qk_norm_rotate_bwd`` check shapes and
dtypes, allocate what is not given, call the C entry point on torch's current
stream of the tensors' device and raise ``lsh.LshError`` on a non-zero status.
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass, replace

import torch

from . import lsh

# Every symbol include/lsh_qk.h declares.
EXPORTED = ("lsh_qk_workspace_bytes", "lsh_qk_norm_rotate_fwd", "lsh_qk_norm_rotate_bwd")


class QkConfigC(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("T", "L", "x_stride", "dx_stride")] + \
               [(n, ctypes.c_int32) for n in ("Hq", "Hk", "d", "rot", "interleaved", "gain_per_head")] + \
               [("eps", ctypes.c_float)]


_lib = None


def lib() -> ctypes.CDLL:
    """lsh.lib() with this header's signatures."""
    global _lib
    if _lib is None:
        L, P, C = lsh.lib(), ctypes.c_void_p, ctypes.POINTER(QkConfigC)
        L.lsh_qk_workspace_bytes.argtypes, L.lsh_qk_workspace_bytes.restype = [C], ctypes.c_size_t
        L.lsh_qk_norm_rotate_fwd.argtypes = [C, ctypes.c_int] + [P] * 8
        L.lsh_qk_norm_rotate_bwd.argtypes = [C, ctypes.c_int] + [P] * 11 + [ctypes.c_size_t, P]
        L.lsh_qk_norm_rotate_fwd.restype = L.lsh_qk_norm_rotate_bwd.restype = ctypes.c_int
        _lib = L
    return _lib


@dataclass(frozen=True)
class QkConfig:
    """T tokens of Hq query heads and Hk key heads (0: shared QK).  L > 0 lays the results out
    [T/L][H][L][64] (the attention's layout), L = 0 [T][H][64]."""
    T: int
    Hq: int
    Hk: int = 0
    L: int = 0
    rot: int = 64
    interleaved: bool = False
    gain_per_head: bool = False
    eps: float = 1e-6
    d: int = 64
    x_stride: int = 0
    dx_stride: int = 0

    def c(self) -> QkConfigC:
        return QkConfigC(self.T, self.L, self.x_stride, self.dx_stride, self.Hq, self.Hk, self.d, self.rot,
                         int(bool(self.interleaved)), int(bool(self.gain_per_head)), self.eps)

    def ref(self):
        """A reference to the C structure, made once: the configuration is frozen."""
        c = self.__dict__.get("_c")
        if c is None:
            c = self.c()
            object.__setattr__(self, "_c", c)
        return ctypes.byref(c)

    def out_shape(self, H: int) -> tuple:
        return (self.T // self.L, H, self.L, self.d) if self.L > 0 else (self.T, H, self.d)

    def gain_shape(self, H: int) -> tuple:
        return (H, self.d) if self.gain_per_head else (self.d,)


def qk_workspace_bytes(cfg: QkConfig) -> int:
    return int(lib().lsh_qk_workspace_bytes(cfg.ref()))


def _token_rows(t: torch.Tensor, T: int, width: int, name: str, stride: int) -> int:
    """Stride between the rows of t, which holds T rows of at least `width` elements (0: packed)."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if t.dim() != 2 or t.shape[0] != T or t.shape[1] < width:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected ({T}, {width} or more)")
    if stride == 0 and t.shape[1] == width and t.is_contiguous():
        return 0
    if t.stride(1) != 1:
        raise ValueError(f"{name}'s rows must be contiguous")
    own = t.stride(0) if T > 1 else stride  # of a single row any
    if T > 1 and own < width:  # also 0, one row for all tokens, which the C call would take for packed rows
        raise ValueError(f"{name} has row stride {own}, its rows have {width} elements")
    if stride not in (0, own):
        raise ValueError(f"{name} has row stride {own}, the configuration {stride}")
    return own


def _check_inputs(cfg: QkConfig, x, gain_q, gain_k, freq, pos) -> QkConfig:
    stride = _token_rows(x, cfg.T, (cfg.Hq + cfg.Hk) * cfg.d, "x", cfg.x_stride)
    if stride != cfg.x_stride:
        cfg = replace(cfg, x_stride=stride)
    lsh._need(gain_q, cfg.gain_shape(cfg.Hq), torch.float32, "gain_q")
    if cfg.Hk:
        if gain_k is None:
            raise ValueError("gain_k is required with key heads")
        lsh._need(gain_k, cfg.gain_shape(cfg.Hk), torch.float32, "gain_k")
    lsh._need(freq, (cfg.rot // 2,), torch.float32, "freq")
    if pos is not None:
        lsh._need(pos, (cfg.T,), torch.int32, "pos")
    dev = x.device
    for name, t in (("gain_q", gain_q), ("gain_k", gain_k), ("freq", freq), ("pos", pos)):
        if t is not None and t.device != dev:
            raise ValueError(f"{name} is on {t.device}, x on {dev}")
    return cfg


def _out(t, shape, dtype, x, name):
    if t is None:
        return torch.empty(shape, dtype=dtype, device=x.device)
    lsh._need(t, shape, dtype, name)
    if t.device != x.device:
        raise ValueError(f"{name} is on {t.device}, x on {x.device}")
    return t


def lsh_qk_norm_rotate_fwd(cfg: QkConfig, x, gain_q, gain_k, freq, pos=None, q=None, k=None):
    """(q, k) of x [T, (Hq + Hk) * 64 or more] (lsh_qk_norm_rotate_fwd); k is None without key heads."""
    cfg = _check_inputs(cfg, x, gain_q, gain_k, freq, pos)
    q = _out(q, cfg.out_shape(cfg.Hq), x.dtype, x, "q")
    k = _out(k, cfg.out_shape(cfg.Hk), x.dtype, x, "k") if cfg.Hk else None
    p = lsh._ptr
    with lsh.on_device(x.device):
        lsh._check("lsh_qk_norm_rotate_fwd",
                   lib().lsh_qk_norm_rotate_fwd(cfg.ref(), lsh._dtype_code(x), p(x), p(gain_q), p(gain_k),
                                                p(freq), p(pos), p(q), p(k), lsh._stream(x.device)))
    return q, k


def lsh_qk_norm_rotate_bwd(cfg: QkConfig, x, gain_q, gain_k, freq, pos, dq, dk=None, dx=None, dgain_q=None,
                           dgain_k=None, workspace=None):
    """(dx, dgain_q, dgain_k), fp32, from the fp32 gradients of q and k (lsh_qk_norm_rotate_bwd)."""
    cfg = _check_inputs(cfg, x, gain_q, gain_k, freq, pos)
    width = (cfg.Hq + cfg.Hk) * cfg.d
    if dq is None:
        raise ValueError("dq is required")
    dq = _out(dq, cfg.out_shape(cfg.Hq), torch.float32, x, "dq")
    if cfg.Hk and dk is None:
        raise ValueError("dk is required with key heads")
    dk = _out(dk, cfg.out_shape(cfg.Hk), torch.float32, x, "dk") if cfg.Hk else None
    if dx is None:
        dx = torch.empty((cfg.T, width), dtype=torch.float32, device=x.device)
    if dx.dtype != torch.float32 or dx.device != x.device:
        raise ValueError(f"dx must be float32 on {x.device}")
    stride = _token_rows(dx, cfg.T, width, "dx", cfg.dx_stride)
    if stride != cfg.dx_stride:
        cfg = replace(cfg, dx_stride=stride)
    dgain_q = _out(dgain_q, cfg.gain_shape(cfg.Hq), torch.float32, x, "dgain_q")
    dgain_k = _out(dgain_k, cfg.gain_shape(cfg.Hk), torch.float32, x, "dgain_k") if cfg.Hk else None
    if workspace is None:
        workspace = torch.empty(max(qk_workspace_bytes(cfg), 256), dtype=torch.uint8, device=x.device)
    lsh._need_workspace(workspace, x.device)
    p = lsh._ptr
    with lsh.on_device(x.device):
        lsh._check("lsh_qk_norm_rotate_bwd",
                   lib().lsh_qk_norm_rotate_bwd(cfg.ref(), lsh._dtype_code(x), p(x), p(gain_q), p(gain_k),
                                                p(freq), p(pos), p(dq), p(dk), p(dx), p(dgain_q), p(dgain_k),
                                                p(workspace), workspace.numel(), lsh._stream(x.device)))
    return dx, dgain_q, dgain_k
