"""Thin Python binding of include/lsh_cache.h: a paged cache of key and value
rows and attention of new tokens over it.

``Pages`` holds the pool, ``Sequences`` says which rows are whose;
``lsh_cache_write``, ``lsh_cache_read`` and ``lsh_cache_attn_fwd`` check shapes
and dtypes, call the C entry point on torch's current stream of the tensors'
device and raise ``lsh.LshError`` on a non-zero status.
"""
from __future__ import annotations

import ctypes
import math
from dataclasses import dataclass, replace

import torch

from . import lsh

# Every symbol include/lsh_cache.h declares.
EXPORTED = ("lsh_cache_workspace_bytes", "lsh_cache_write", "lsh_cache_read", "lsh_cache_attn_fwd")
TYPES = {"bf16": 0, "e4m3": 1, "e2m1": 2}
ROW_BYTES = {"bf16": 128, "e4m3": 64, "e2m1": 32}


class CacheConfigC(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("T", "q_stride", "k_stride", "v_stride")] + \
               [(n, ctypes.c_int32) for n in ("n_seq", "H", "Hkv", "d", "page", "n_pages", "max_pages", "type",
                                              "shared_qk", "max_new")] + \
               [("scale", ctypes.c_float), ("self_mask", ctypes.c_float)]


class CachePagesC(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k", "v", "k_scale", "v_scale", "k_inv")]


class CacheSeqsC(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("first", "length", "table")]


_lib = None


def lib() -> ctypes.CDLL:
    """lsh.lib() with this header's signatures."""
    global _lib
    if _lib is None:
        L, P, I = lsh.lib(), ctypes.c_void_p, ctypes.c_int
        C = ctypes.POINTER(CacheConfigC)
        head = [C, I, ctypes.POINTER(CachePagesC), ctypes.POINTER(CacheSeqsC)]
        L.lsh_cache_workspace_bytes.argtypes, L.lsh_cache_workspace_bytes.restype = [C], ctypes.c_size_t
        L.lsh_cache_write.argtypes = L.lsh_cache_read.argtypes = head + [P, P, P]
        L.lsh_cache_attn_fwd.argtypes = head + [P, P, P, P, ctypes.c_size_t, P]
        for fn in (L.lsh_cache_write, L.lsh_cache_read, L.lsh_cache_attn_fwd):
            fn.restype = I
        _lib = L
    return _lib


@dataclass(frozen=True)
class CacheConfig:
    """T new tokens of n_seq sequences, H query heads over Hkv key heads, a pool of n_pages pages.
    max_new (most new tokens of one sequence; 0: unknown) only helps to choose kernels."""
    n_seq: int
    T: int
    H: int
    Hkv: int
    n_pages: int
    max_pages: int
    page: int = 64
    type: str = "bf16"
    shared_qk: bool = True
    scale: float | None = None
    self_mask: float = 1e5
    max_new: int = 0
    d: int = 64
    q_stride: int = 0
    k_stride: int = 0
    v_stride: int = 0

    def c(self) -> CacheConfigC:
        scale = 1.0 / math.sqrt(self.d) if self.scale is None else self.scale
        return CacheConfigC(self.T, self.q_stride, self.k_stride, self.v_stride, self.n_seq, self.H, self.Hkv, self.d,
                            self.page, self.n_pages, self.max_pages, TYPES[self.type], int(bool(self.shared_qk)),
                            self.max_new, scale, self.self_mask)

    def ref(self):
        """A reference to the C structure, made once: the configuration is frozen."""
        c = self.__dict__.get("_c")
        if c is None:
            c = self.c()
            object.__setattr__(self, "_c", c)
        return ctypes.byref(c)

    def strides(self, **own) -> "CacheConfig":
        """This configuration with the tensors' token strides."""
        own = {k: v for k, v in own.items() if v != getattr(self, k)}
        return replace(self, **own) if own else self


@dataclass(frozen=True)
class Pages:
    """The pool: k, v uint8 [n_pages, Hkv, page, row bytes], k_scale, v_scale uint8 [n_pages, Hkv, page, 2]
    (None for bf16), k_inv fp32 [n_pages, Hkv, page] (None unless shared_qk)."""
    k: torch.Tensor
    v: torch.Tensor
    k_scale: torch.Tensor | None = None
    v_scale: torch.Tensor | None = None
    k_inv: torch.Tensor | None = None

    @staticmethod
    def empty(cfg: CacheConfig, device) -> "Pages":
        slots = (cfg.n_pages, cfg.Hkv, cfg.page)

        def new(*more, dtype=torch.uint8):
            return torch.empty(slots + more, dtype=dtype, device=device)

        scales = [None, None] if cfg.type == "bf16" else [new(2), new(2)]
        return Pages(new(ROW_BYTES[cfg.type]), new(ROW_BYTES[cfg.type]), *scales,
                     new(dtype=torch.float32) if cfg.shared_qk else None)

    def check(self, cfg: CacheConfig) -> None:
        if self.__dict__.get("_checked") is cfg:  # these tensors against this configuration: once
            return
        slots = (cfg.n_pages, cfg.Hkv, cfg.page)
        want = [("k", (ROW_BYTES[cfg.type],), torch.uint8), ("v", (ROW_BYTES[cfg.type],), torch.uint8)]
        if cfg.type != "bf16":
            want += [("k_scale", (2,), torch.uint8), ("v_scale", (2,), torch.uint8)]
        if cfg.shared_qk:
            want += [("k_inv", (), torch.float32)]
        for name, more, dtype in want:
            t = getattr(self, name)
            if t is None:
                raise ValueError(f"the pool has no {name}")
            lsh._need(t, slots + more, dtype, name)
            if t.device != self.k.device:
                raise ValueError(f"{name} is on {t.device}, k on {self.k.device}")
        object.__setattr__(self, "_checked", cfg)

    def c(self) -> CachePagesC:
        return CachePagesC(*[lsh._ptr(t) for t in (self.k, self.v, self.k_scale, self.v_scale, self.k_inv)])


@dataclass(frozen=True)
class Sequences:
    """first [n_seq + 1], length [n_seq], table [n_seq, max_pages], all int32 on the GPU.  What they hold may
    change between calls."""
    first: torch.Tensor
    length: torch.Tensor
    table: torch.Tensor

    def check(self, cfg: CacheConfig, device) -> None:
        checked = self.__dict__.get("_checked")
        if checked is not None and checked[0] is cfg and checked[1] == device:
            return
        for name, shape in (("first", (cfg.n_seq + 1,)), ("length", (cfg.n_seq,)), ("table", (cfg.n_seq, cfg.max_pages))):
            t = getattr(self, name)
            lsh._need(t, shape, torch.int32, name)
            if t.device != device:
                raise ValueError(f"{name} is on {t.device}, the pages on {device}")
        object.__setattr__(self, "_checked", (cfg, device))

    def c(self) -> CacheSeqsC:
        return CacheSeqsC(lsh._ptr(self.first), lsh._ptr(self.length), lsh._ptr(self.table))


def _rows(t: torch.Tensor, cfg: CacheConfig, H: int, name: str, stride: int, device, dtype=None) -> int:
    """Token stride of rows t [T, H, 64], whose heads are next to each other (0: packed)."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the pages on {device}")
    if t.shape != (cfg.T, H, cfg.d):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {(cfg.T, H, cfg.d)}")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if stride == 0 and t.is_contiguous():
        return 0
    if t.stride(2) != 1 or (H > 1 and t.stride(1) != cfg.d):
        raise ValueError(f"{name}'s heads must be contiguous")
    own = t.stride(0) if cfg.T > 1 else stride  # of a single row any
    if cfg.T > 1 and own < H * cfg.d:  # also 0, one row for all tokens, which the C call would take for packed rows
        raise ValueError(f"{name} has token stride {own}, its rows have {H * cfg.d} elements")
    if stride not in (0, own):
        raise ValueError(f"{name} has token stride {own}, the configuration {stride}")
    return own


def workspace_bytes(cfg: CacheConfig) -> int:
    return int(lib().lsh_cache_workspace_bytes(cfg.ref()))


def workspace(cfg: CacheConfig, device) -> torch.Tensor:
    """A workspace for lsh_cache_attn_fwd; calls that may overlap need one each."""
    return torch.empty(max(workspace_bytes(cfg), 256), dtype=torch.uint8, device=device)


def lsh_cache_write(cfg: CacheConfig, pages: Pages, seqs: Sequences, k, v) -> None:
    """The new tokens' rows k, v [T, Hkv, 64] into the cache (lsh_cache_write)."""
    pages.check(cfg)
    dev = pages.k.device
    seqs.check(cfg, dev)
    cfg = cfg.strides(k_stride=_rows(k, cfg, cfg.Hkv, "k", cfg.k_stride, dev),
                      v_stride=_rows(v, cfg, cfg.Hkv, "v", cfg.v_stride, dev, k.dtype))
    with lsh.on_device(dev):
        lsh._check("lsh_cache_write",
                   lib().lsh_cache_write(cfg.ref(), lsh._dtype_code(k), ctypes.byref(pages.c()),
                                         ctypes.byref(seqs.c()), lsh._ptr(k), lsh._ptr(v), lsh._stream(dev)))


def lsh_cache_read(cfg: CacheConfig, pages: Pages, seqs: Sequences, dtype: torch.dtype, k=None, v=None):
    """Rows k, v [T, Hkv, 64] of the sequences' last positions, in dtype (lsh_cache_read).  Rows
    outside all sequences are left as they are."""
    pages.check(cfg)
    dev = pages.k.device
    seqs.check(cfg, dev)
    k = torch.empty((cfg.T, cfg.Hkv, cfg.d), dtype=dtype, device=dev) if k is None else k
    v = torch.empty((cfg.T, cfg.Hkv, cfg.d), dtype=dtype, device=dev) if v is None else v
    cfg = cfg.strides(k_stride=_rows(k, cfg, cfg.Hkv, "k", cfg.k_stride, dev, dtype),
                      v_stride=_rows(v, cfg, cfg.Hkv, "v", cfg.v_stride, dev, dtype))
    with lsh.on_device(dev):
        lsh._check("lsh_cache_read",
                   lib().lsh_cache_read(cfg.ref(), lsh._dtype_code(k), ctypes.byref(pages.c()),
                                        ctypes.byref(seqs.c()), lsh._ptr(k), lsh._ptr(v), lsh._stream(dev)))
    return k, v


def lsh_cache_attn_fwd(cfg: CacheConfig, pages: Pages, seqs: Sequences, q, out=None, lse=None, workspace=None):
    """(out [T, H, 64] bf16, lse [T, H] fp32) of the new tokens' queries q (lsh_cache_attn_fwd)."""
    pages.check(cfg)
    dev = pages.k.device
    seqs.check(cfg, dev)
    cfg = cfg.strides(q_stride=_rows(q, cfg, cfg.H, "q", cfg.q_stride, dev, torch.bfloat16))
    if out is None:
        out = torch.empty((cfg.T, cfg.H, cfg.d), dtype=torch.bfloat16, device=dev)
    if lse is None:
        lse = torch.empty((cfg.T, cfg.H), dtype=torch.float32, device=dev)
    lsh._need(out, (cfg.T, cfg.H, cfg.d), torch.bfloat16, "out")
    lsh._need(lse, (cfg.T, cfg.H), torch.float32, "lse")
    if workspace is None:
        workspace = torch.empty(max(workspace_bytes(cfg), 256), dtype=torch.uint8, device=dev)
    lsh._need_workspace(workspace, dev)
    for name, t in (("out", out), ("lse", lse)):
        if t.device != dev:
            raise ValueError(f"{name} is on {t.device}, the pages on {dev}")
    with lsh.on_device(dev):
        lsh._check("lsh_cache_attn_fwd",
                   lib().lsh_cache_attn_fwd(cfg.ref(), lsh.LSH_BF16, ctypes.byref(pages.c()),
                                            ctypes.byref(seqs.c()), lsh._ptr(q), lsh._ptr(out), lsh._ptr(lse),
                                            lsh._ptr(workspace), workspace.numel(), lsh._stream(dev)))
    return out, lse
