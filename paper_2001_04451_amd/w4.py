"""Thin Python binding of include/lsh_w4.h: products with weights of 4 bits.

``lsh_w4_quantize`` and ``lsh_w4_pack`` lay a matrix out once; ``lsh_linear_w4``
multiplies rows by it.  The functions check shapes, dtypes and devices, allocate
what is not given, call the C entry point on torch's current stream of the
tensors' device and raise ``lsh.LshError`` on a non-zero status.
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass

import torch

from . import lsh

# Every symbol include/lsh_w4.h declares.
EXPORTED = ("lsh_w4_weight_bytes", "lsh_w4_workspace_bytes", "lsh_w4_quantize", "lsh_w4_pack", "lsh_w4_unpack",
            "lsh_linear_w4")
TYPES = {"int4": 0, "e2m1": 1}


class W4ConfigC(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("N", "K", "type", "group", "zeros")]


_lib = None


def lib() -> ctypes.CDLL:
    """lsh.lib() with this header's signatures."""
    global _lib
    if _lib is None:
        L, P, I, C = lsh.lib(), ctypes.c_void_p, ctypes.c_int, ctypes.POINTER(W4ConfigC)
        n, size, f = ctypes.c_int64, ctypes.c_size_t, ctypes.c_float
        L.lsh_w4_weight_bytes.argtypes, L.lsh_w4_weight_bytes.restype = [C], size
        L.lsh_w4_workspace_bytes.argtypes, L.lsh_w4_workspace_bytes.restype = [C, n], size
        L.lsh_w4_quantize.argtypes = [C, I, P, P, P]
        L.lsh_w4_pack.argtypes = [C, P, P, P, P, P]
        L.lsh_w4_unpack.argtypes = [C, I, P, P, P]
        L.lsh_linear_w4.argtypes = [C, n, P, n, P, P, P, f, I, P, P, P, size, P]
        for fn in (L.lsh_w4_quantize, L.lsh_w4_pack, L.lsh_w4_unpack, L.lsh_linear_w4):
            fn.restype = I
        _lib = L
    return _lib


@dataclass(frozen=True)
class W4Config:
    """A matrix of N outputs x K inputs in 4 bits.  type "int4": a bf16 scale, and with ``zeros`` a zero point,
    for each ``group`` of 32, 64 or 128 inputs; "e2m1": a power-of-two scale for each 32."""
    N: int
    K: int
    type: str = "int4"
    group: int = 128
    zeros: bool = False

    def c(self) -> W4ConfigC:
        for name, n in (("N", self.N), ("K", self.K), ("group", self.group)):
            if not 0 <= n < 1 << 31:  # a c_int32 would take it modulo 2^32
                raise ValueError(f"{name} = {n} is out of range")
        return W4ConfigC(self.N, self.K, TYPES[self.type], self.group, int(bool(self.zeros)))

    def ref(self):
        """A reference to the C structure, made once: the configuration is frozen."""
        c = self.__dict__.get("_c")
        if c is None:
            c = self.c()
            object.__setattr__(self, "_c", c)
        return ctypes.byref(c)

    def groups(self) -> int:
        return -(-self.K // self.group)

    def bytes(self) -> int:
        """weight_bytes(), asked once."""
        n = self.__dict__.get("_bytes")
        if n is None:
            n = weight_bytes(self)
            object.__setattr__(self, "_bytes", n)
        return n


def weight_bytes(cfg: W4Config) -> int:
    return int(lib().lsh_w4_weight_bytes(cfg.ref()))


def workspace_bytes(cfg: W4Config, M: int) -> int:
    return int(lib().lsh_w4_workspace_bytes(cfg.ref(), M))


def workspace(cfg: W4Config, M: int, device) -> torch.Tensor:
    """A workspace for lsh_linear_w4 of up to M rows; calls that may overlap need one each."""
    # Fewer rows may need more, being split.  Tiles have a multiple of 64 rows, between which the need grows.
    n = max([workspace_bytes(cfg, M)] + [workspace_bytes(cfg, m) for m in range(64, M, 64)])
    return torch.empty(max(n, 256), dtype=torch.uint8, device=device)


def _packed(cfg: W4Config, packed, device) -> torch.Tensor:
    n = cfg.bytes()
    if packed is None:
        return torch.empty(max(n, 256), dtype=torch.uint8, device=device)
    if packed.dtype != torch.uint8 or packed.numel() < n or not packed.is_contiguous():
        raise ValueError(f"packed has {packed.numel()} elements of {packed.dtype}, expected {n} of uint8 or more, "
                         "next to each other")
    if packed.device != device:
        raise ValueError(f"packed is on {packed.device}, the tensors on {device}")
    return packed


def lsh_w4_quantize(cfg: W4Config, w, packed=None) -> torch.Tensor:
    """The packed weights of a matrix w [N, K] in fp32 or bf16 (lsh_w4_quantize)."""
    lsh._need(w, (cfg.N, cfg.K), None, "w")
    code = lsh._dtype_code(w)
    packed = _packed(cfg, packed, w.device)
    with lsh.on_device(w.device):
        lsh._check("lsh_w4_quantize",
                   lib().lsh_w4_quantize(cfg.ref(), code, lsh._ptr(w), lsh._ptr(packed), lsh._stream(w.device)))
    return packed


def lsh_w4_pack(cfg: W4Config, codes, scales, zeros=None, packed=None) -> torch.Tensor:
    """The packed weights of codes uint8 [N, K/2], scales [N, groups] (bf16, or uint8 for e2m1) and, with
    cfg.zeros, zero points uint8 [N, groups] (lsh_w4_pack)."""
    lsh._need(codes, (cfg.N, cfg.K // 2), torch.uint8, "codes")
    lsh._need(scales, (cfg.N, cfg.groups()), torch.uint8 if cfg.type == "e2m1" else torch.bfloat16, "scales")
    if (zeros is not None) != bool(cfg.zeros):
        raise ValueError("zeros has to be given exactly where the configuration has zero points")
    if zeros is not None:
        lsh._need(zeros, (cfg.N, cfg.groups()), torch.uint8, "zeros")
    for name, t in (("scales", scales), ("zeros", zeros)):
        if t is not None and t.device != codes.device:
            raise ValueError(f"{name} is on {t.device}, codes on {codes.device}")
    packed = _packed(cfg, packed, codes.device)
    with lsh.on_device(codes.device):
        lsh._check("lsh_w4_pack",
                   lib().lsh_w4_pack(cfg.ref(), lsh._ptr(codes), lsh._ptr(scales), lsh._ptr(zeros), lsh._ptr(packed),
                                     lsh._stream(codes.device)))
    return packed


def lsh_w4_unpack(cfg: W4Config, packed, dtype: torch.dtype = torch.float32, w=None) -> torch.Tensor:
    """The matrix w [N, K] that packed weights stand for, in fp32 (exact) or bf16 (lsh_w4_unpack)."""
    if not packed.is_cuda:
        raise ValueError("packed must be a GPU tensor")
    packed = _packed(cfg, packed, packed.device)
    if w is None:
        w = torch.empty((cfg.N, cfg.K), dtype=dtype, device=packed.device)
    lsh._need(w, (cfg.N, cfg.K), dtype, "w")
    if w.device != packed.device:
        raise ValueError(f"w is on {w.device}, packed on {packed.device}")
    with lsh.on_device(packed.device):
        lsh._check("lsh_w4_unpack",
                   lib().lsh_w4_unpack(cfg.ref(), lsh._dtype_code(w), lsh._ptr(packed), lsh._ptr(w),
                                       lsh._stream(packed.device)))
    return w


def _row_stride(a, K: int) -> int:
    """Elements between the rows of a [M, K] (0: packed)."""
    if not a.is_cuda:
        raise ValueError("a must be a GPU tensor")
    shape = a.shape
    if len(shape) != 2 or shape[1] != K or shape[0] < 1:
        raise ValueError(f"a has shape {tuple(shape)}, expected (1 or more, {K})")
    if a.dtype != torch.bfloat16:
        raise ValueError(f"a has dtype {a.dtype}, expected torch.bfloat16")
    if a.is_contiguous():
        return 0
    own = a.stride(0)
    if a.stride(1) != 1:
        raise ValueError("a's rows must be contiguous")
    if shape[0] == 1:  # of a single row any
        return 0
    if own < K:  # also 0, one row for all, which the C call would take for packed rows
        raise ValueError(f"a has row stride {own}, its rows have {K} elements")
    return own


def _beside(t, shape, dtype, dev, name) -> int | None:
    """The address of t, contiguous and on a's device."""
    if t is None:
        return None
    lsh._need(t, shape, dtype, name)
    if t.device != dev:
        raise ValueError(f"{name} is on {t.device}, a on {dev}")
    return t.data_ptr()


def lsh_linear_w4(cfg: W4Config, a, packed, bias=None, resid=None, sign: float = 1.0, relu: bool = False,
                  dtype: torch.dtype = torch.float32, out=None, workspace=None) -> torch.Tensor:
    """resid + sign (a W^T + bias) in fp32, or with dtype bfloat16 bf16(a W^T + bias), relu before the rounding
    with ``relu`` (lsh_linear_w4).  a [M, K] bf16, its rows at any stride that is a multiple of 8."""
    if packed is None:
        raise ValueError("packed is required")
    if sign != 1.0 and dtype == torch.bfloat16:
        raise ValueError("sign goes with float32")
    stride = _row_stride(a, cfg.K)
    dev, shape = a.device, (a.shape[0], cfg.N)
    packed = _packed(cfg, packed, dev)
    f32 = dtype == torch.float32
    if not f32 and dtype != torch.bfloat16:
        raise TypeError(f"unsupported dtype {dtype}; use float32 or bfloat16")
    if out is None:
        out = a.new_empty(shape, dtype=dtype)
        to = out.data_ptr()
    else:
        to = _beside(out, shape, dtype, dev, "out")
    bias = _beside(bias, (cfg.N,), torch.float32, dev, "bias")
    resid = _beside(resid, shape, torch.float32, dev, "resid")
    if workspace is None:
        n = workspace_bytes(cfg, shape[0])
        workspace = torch.empty(n, dtype=torch.uint8, device=dev) if n else None
    else:
        lsh._need_workspace(workspace, dev)
    with lsh.on_device(dev):
        lsh._check("lsh_linear_w4",
                   lib().lsh_linear_w4(cfg.ref(), shape[0], a.data_ptr(), stride, packed.data_ptr(), bias, resid, sign,
                                       bool(relu), to if f32 else None, None if f32 else to, lsh._ptr(workspace),
                                       0 if workspace is None else workspace.numel(), lsh._stream(dev)))
    return out
