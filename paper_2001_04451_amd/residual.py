"""Thin Python binding of include/lsh_residual.h: the step between two blocks.

A block's output is normed, gated, scaled and added to the residual stream, and
the stream is normed for the next block (``lsh_residual_norm_fwd``), with the
gradients of all of it (``lsh_residual_norm_bwd``).  The functions check shapes,
dtypes and devices, allocate what is not given, call the C entry point on torch's
current stream of the tensors' device and raise ``lsh.LshError`` on a non-zero
status.
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass, replace

import torch

from . import lsh

# Every symbol include/lsh_residual.h declares.
EXPORTED = ("lsh_residual_workspace_bytes", "lsh_residual_norm_fwd", "lsh_residual_norm_bwd")
NORMS = {"rms": 0, "layer": 1}
GATES = {"none": 0, "linear": 1, "sigmoid": 2}
WEIGHTS = ("scale", "post_g", "post_b", "pre_g", "pre_b")
GRADS = ("dx", "df", "dgate", "dscale", "dpost_g", "dpost_b", "dpre_g", "dpre_b")


class ResidualConfigC(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("T", "f_stride", "gate_stride")] + \
               [(n, ctypes.c_int32) for n in ("D", "norm", "post", "pre", "gate")] + \
               [("alpha", ctypes.c_float), ("eps", ctypes.c_float)]


class ResidualWeightsC(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in WEIGHTS]


class ResidualGradsC(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in GRADS]


_lib = None


def lib() -> ctypes.CDLL:
    """lsh.lib() with this header's signatures."""
    global _lib
    if _lib is None:
        L, P, I = lsh.lib(), ctypes.c_void_p, ctypes.c_int
        C, W, G = (ctypes.POINTER(t) for t in (ResidualConfigC, ResidualWeightsC, ResidualGradsC))
        L.lsh_residual_workspace_bytes.argtypes, L.lsh_residual_workspace_bytes.restype = [C], ctypes.c_size_t
        L.lsh_residual_norm_fwd.argtypes = [C, I, P, P, P, W, P, P, P]
        L.lsh_residual_norm_bwd.argtypes = [C, I, P, P, P, W, P, P, G, P, ctypes.c_size_t, P]
        L.lsh_residual_norm_fwd.restype = L.lsh_residual_norm_bwd.restype = I
        _lib = L
    return _lib


@dataclass(frozen=True)
class ResidualConfig:
    """T rows of D values.  ``post``: the block's output is normed; ``pre``: the stream is normed for the next block;
    ``norm`` "rms" or "layer"; ``gate`` "none", "linear" or "sigmoid"; ``alpha`` multiplies the branch."""
    T: int
    D: int
    norm: str = "rms"
    post: bool = True
    pre: bool = True
    gate: str = "none"
    alpha: float = 1.0
    eps: float = 1e-6
    f_stride: int = 0
    gate_stride: int = 0

    def c(self) -> ResidualConfigC:
        if not 0 <= self.D < 1 << 31:  # a c_int32 would take it modulo 2^32
            raise ValueError(f"D = {self.D} is out of range")
        return ResidualConfigC(self.T, self.f_stride, self.gate_stride, self.D, NORMS[self.norm], int(bool(self.post)),
                               int(bool(self.pre)), GATES[self.gate], self.alpha, self.eps)

    def ref(self):
        """A reference to the C structure, made once: the configuration is frozen."""
        c = self.__dict__.get("_c")
        if c is None:
            c = self.c()
            object.__setattr__(self, "_c", c)
        return ctypes.byref(c)


@dataclass(frozen=True)
class ResidualWeights:
    """fp32 [D] each: ``scale`` of the branch (None: 1), gains and biases of the two norms (biases None: 0)."""
    scale: torch.Tensor | None = None
    post_g: torch.Tensor | None = None
    post_b: torch.Tensor | None = None
    pre_g: torch.Tensor | None = None
    pre_b: torch.Tensor | None = None

    def check(self, cfg: ResidualConfig, device) -> None:
        shape, f32 = (cfg.D,), torch.float32
        for t in (self.scale, self.post_g, self.post_b, self.pre_g, self.pre_b):
            # at every call: a parameter's storage may be exchanged for one of another type
            if t is not None and (t.dtype is not f32 or t.device != device or t.shape != shape or not t.is_contiguous()):
                self._refuse(cfg, device)
        if (self.post_g is not None) != bool(cfg.post) or (self.pre_g is not None) != bool(cfg.pre) or \
                (self.post_b is not None and not cfg.post) or (self.pre_b is not None and not cfg.pre):
            self._refuse(cfg, device)

    def _refuse(self, cfg: ResidualConfig, device) -> None:
        """Raises what check() has found, by name."""
        for name in WEIGHTS:
            t = getattr(self, name)
            if t is None:
                continue
            lsh._need(t, (cfg.D,), torch.float32, name)
            if t.device != device:
                raise ValueError(f"{name} is on {t.device}, the rows on {device}")
        for on, name in ((cfg.post, "post"), (cfg.pre, "pre")):
            if on and getattr(self, name + "_g") is None:
                raise ValueError(f"{name}_g is required with {name}")
            if not on and (getattr(self, name + "_g") is not None or getattr(self, name + "_b") is not None):
                raise ValueError(f"{name}_g and {name}_b go with {name}")

    def ref(self):
        p = lsh._ptr
        return ctypes.byref(ResidualWeightsC(p(self.scale), p(self.post_g), p(self.post_b), p(self.pre_g),
                                             p(self.pre_b)))


def workspace_bytes(cfg: ResidualConfig) -> int:
    return int(lib().lsh_residual_workspace_bytes(cfg.ref()))


def _rows(t, cfg: ResidualConfig, name: str, stride: int) -> int:
    """Stride between the rows of t [T, D] (0: packed)."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if t.shape != (cfg.T, cfg.D):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {(cfg.T, cfg.D)}")
    if stride == 0 and t.is_contiguous():
        return 0
    if t.stride(1) != 1:
        raise ValueError(f"{name}'s rows must be contiguous")
    own = t.stride(0) if cfg.T > 1 else stride  # of a single row any
    if cfg.T > 1 and own < cfg.D:  # also 0, one row for all, which the C call would take for packed rows
        raise ValueError(f"{name} has row stride {own}, its rows have {cfg.D} elements")
    if stride not in (0, own):
        raise ValueError(f"{name} has row stride {own}, the configuration {stride}")
    return own


def _inputs(cfg: ResidualConfig, f, gate, weights, like):
    """(configuration with the rows' strides, dtype code or None, device)."""
    if f is None and (gate is not None or cfg.post or weights.scale is not None):
        raise ValueError("without f there is no gate, scale or post")
    if (gate is not None) != (cfg.gate != "none"):
        raise ValueError("gate has to be given exactly where the configuration has one")
    dev = (like if f is None else f).device
    weights.check(cfg, dev)
    if f is None:
        return cfg, None, dev
    code, f_stride, gate_stride = lsh._dtype_code(f), _rows(f, cfg, "f", cfg.f_stride), cfg.gate_stride
    if gate is not None:
        gate_stride = _rows(gate, cfg, "gate", gate_stride)
        if gate.dtype != f.dtype or gate.device != dev:
            raise ValueError(f"gate is {gate.dtype} on {gate.device}, f {f.dtype} on {dev}")
    if f_stride != cfg.f_stride or gate_stride != cfg.gate_stride:
        cfg = replace(cfg, f_stride=f_stride, gate_stride=gate_stride)
    return cfg, code, dev


def _take(t, shape, dtype, dev, name, make=True):
    if t is None:
        return torch.empty(shape, dtype=dtype, device=dev) if make else None
    lsh._need(t, shape, dtype, name)
    if t.device != dev:
        raise ValueError(f"{name} is on {t.device}, the rows on {dev}")
    return t


def lsh_residual_norm_fwd(cfg: ResidualConfig, x, f, gate, weights: ResidualWeights, y=None, z=None,
                          dtype: torch.dtype | None = None):
    """(y [T, D] fp32, z [T, D] or None without cfg.pre) of the stream x fp32 (None: 0), the block's output f and its
    gate (lsh_residual_norm_fwd).  z has f's dtype; without f (the norm before the first block) ``dtype``, bfloat16 if
    it is None."""
    if f is None and x is None:
        raise ValueError("without f, x is required")
    cfg, code, dev = _inputs(cfg, f, gate, weights, x)
    shape = (cfg.T, cfg.D)
    own = f.dtype if f is not None else (dtype or torch.bfloat16)
    if dtype is not None and dtype != own:
        raise ValueError(f"z has f's dtype {own}, not {dtype}")
    if code is None:
        code = lsh._dtype_code(torch.empty(0, dtype=own))
    x = _take(x, shape, torch.float32, dev, "x", False)
    y = x.new_empty(shape) if y is None and x is not None else _take(y, shape, torch.float32, dev, "y")
    if z is not None and not cfg.pre:
        raise ValueError("z goes with pre")
    if not cfg.pre:
        z = None
    elif z is None and f is not None:
        z = f.new_empty(shape)
    else:
        z = _take(z, shape, own, dev, "z")
    p = lsh._ptr
    with lsh.on_device(dev):
        lsh._check("lsh_residual_norm_fwd",
                   lib().lsh_residual_norm_fwd(cfg.ref(), code, p(x), p(f), p(gate), weights.ref(), p(y), p(z),
                                               lsh._stream(dev)))
    return y, z


def lsh_residual_norm_bwd(cfg: ResidualConfig, y, f, gate, weights: ResidualWeights, dy, dz, grads=None,
                          workspace=None) -> dict:
    """The fp32 gradients by name (GRADS; None where the call has no such input or weight), from the forward's y, f and
    gate and the fp32 gradients of y (None: 0) and z (lsh_residual_norm_bwd).  ``grads``: tensors to write to."""
    if (dz is not None) != bool(cfg.pre) or (dy is None and dz is None):
        raise ValueError("dz has to be given exactly with pre, and dy without it")
    cfg, code, dev = _inputs(cfg, f, gate, weights, dy if dz is None else dz)
    shape = (cfg.T, cfg.D)
    if cfg.pre and y is None:
        raise ValueError("y is required with pre")
    y = _take(y, shape, torch.float32, dev, "y", False)
    dy = _take(dy, shape, torch.float32, dev, "dy", False)
    dz = _take(dz, shape, torch.float32, dev, "dz", False)
    there = {"dx": True, "df": f is not None, "dgate": gate is not None}
    there.update({"d" + n: getattr(weights, n) is not None for n in WEIGHTS})
    given = grads or {}
    if any(n not in there or (t is not None and not there[n]) for n, t in given.items()):
        raise ValueError("grads holds a tensor that is no gradient of this call")
    out = {n: _take(given.get(n), shape if i < 3 else (cfg.D,), torch.float32, dev, n) if there[n] else None
           for i, n in enumerate(GRADS)}
    if workspace is None:
        workspace = torch.empty(max(workspace_bytes(cfg), 256), dtype=torch.uint8, device=dev)
    lsh._need_workspace(workspace, dev)
    p = lsh._ptr
    with lsh.on_device(dev):
        lsh._check("lsh_residual_norm_bwd",
                   lib().lsh_residual_norm_bwd(cfg.ref(), lsh.LSH_BF16 if code is None else code, p(y), p(f), p(gate),
                                               weights.ref(), p(dy), p(dz),
                                               ctypes.byref(ResidualGradsC(*[p(out[n]) for n in GRADS])),
                                               p(workspace), workspace.numel(), lsh._stream(dev)))
    return out
