"""The C ABI and bindings of the 4-bit weights, of the step between two blocks and of the cache's append without a GPU:
exported symbols, workspaces, and every refusal before any HIP call."""
import copy
import ctypes
import os
import pickle
import re

import pytest
import torch

from paper_2001_04451_amd import cache, lsh, qk, residual, w4

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = ctypes.c_void_p(0x1000)  # never dereferenced: every call below fails validation
ODD = ctypes.c_void_p(0x1008)
INVALID, UNSUPPORTED = lsh.LSH_ERR_INVALID, lsh.LSH_ERR_UNSUPPORTED
BIG = 1 << 40


@pytest.fixture(scope="module")
def built():
    if not os.path.exists(lsh.LIB_PATH):
        pytest.skip("liblsh.so not built (run __graft_entry__.build())")


@pytest.mark.parametrize("module,header", [(w4, "lsh_w4.h"), (residual, "lsh_residual.h")])
def test_header_symbols_exported(built, module, header):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
    assert set(re.findall(r"\b(lsh_[a-z0-9_]+)\s*\(", text)) == set(module.EXPORTED)
    for name in module.EXPORTED:
        assert hasattr(module.lib(), name)


# ----------------------------------------------------------------------------
# 4-bit weights


def _w4(**kw):
    base = dict(N=48, K=256)
    base.update(kw)
    return w4.W4Config(**base)


BAD_W4 = [(dict(N=0), INVALID), (dict(K=0), INVALID), (dict(group=16), INVALID), (dict(group=0), INVALID),
          (dict(group=256), INVALID), (dict(type="e2m1"), INVALID), (dict(type="e2m1", group=64), INVALID),
          (dict(type="e2m1", group=32, zeros=True), INVALID), (dict(K=40), UNSUPPORTED), (dict(K=(1 << 17) + 32), UNSUPPORTED),
          (dict(N=(1 << 22) + 1), UNSUPPORTED), (dict(N=1 << 22, K=1 << 17), UNSUPPORTED)]


def _w4_calls(c, M=4, dtype=1):
    L, r = w4.lib(), ctypes.byref(c) if c is not None else None
    zeros = FAKE if c is not None and c.zeros else None
    return (L.lsh_w4_quantize(r, dtype, FAKE, FAKE, None), L.lsh_w4_pack(r, FAKE, FAKE, zeros, FAKE, None),
            L.lsh_w4_unpack(r, dtype, FAKE, FAKE, None),
            L.lsh_linear_w4(r, M, FAKE, 0, FAKE, None, None, 1.0, 0, FAKE, None, FAKE, BIG, None))


@pytest.mark.parametrize("bad,status", BAD_W4)
def test_w4_config_refused(built, bad, status):
    cfg = _w4(**bad)
    assert w4.weight_bytes(cfg) == 0 and w4.workspace_bytes(cfg, 4) == 0
    assert set(_w4_calls(cfg.c())) == {status}


def test_w4_arguments_refused(built):
    L, cfg = w4.lib(), _w4(zeros=True)
    c = cfg.c()
    assert set(_w4_calls(None)) == {INVALID}
    for type_ in (-1, 2):
        bad = cfg.c()
        bad.type = type_
        assert set(_w4_calls(bad)) == {INVALID}
    r = ctypes.byref(c)
    for p in (None, ODD):
        assert L.lsh_w4_quantize(r, 1, p, FAKE, None) == L.lsh_w4_quantize(r, 1, FAKE, p, None) == INVALID
        assert L.lsh_w4_unpack(r, 1, p, FAKE, None) == L.lsh_w4_unpack(r, 1, FAKE, p, None) == INVALID
        for i in range(4):  # codes, scales, zeros, packed
            assert L.lsh_w4_pack(r, *[p if j == i else FAKE for j in range(4)], None) == INVALID, i
    plain = ctypes.byref(_w4().c())
    assert L.lsh_w4_pack(plain, FAKE, FAKE, FAKE, FAKE, None) == INVALID  # zero points that the type has not
    assert L.lsh_w4_quantize(r, 3, FAKE, FAKE, None) == L.lsh_w4_unpack(r, 3, FAKE, FAKE, None) == INVALID
    assert L.lsh_w4_quantize(r, 1, FAKE, ctypes.c_void_p(0x1010), None) == INVALID  # packed on 256 bytes

    def linear(M=4, a=FAKE, stride=0, packed=FAKE, bias=None, resid=None, sign=1.0, relu=0, f32=FAKE, b16=None, ws=FAKE, n=BIG):
        return L.lsh_linear_w4(r, M, a, stride, packed, bias, resid, sign, relu, f32, b16, ws, n, None)

    assert w4.workspace_bytes(cfg, 0) == w4.workspace_bytes(cfg, 1 << 40) == 0
    assert linear(M=0) == linear(M=-3) == INVALID
    assert linear(M=(1 << 24) + 1) == linear(M=1 << 40) == UNSUPPORTED
    assert linear(a=None) == linear(a=ODD) == linear(packed=None) == linear(packed=ctypes.c_void_p(0x1010)) == INVALID
    assert linear(stride=248) == linear(stride=260) == linear(stride=-8) == INVALID
    assert linear(stride=1 << 32) == UNSUPPORTED
    assert linear(f32=None) == linear(b16=FAKE) == linear(f32=ODD) == linear(f32=None, b16=ODD) == INVALID
    assert linear(relu=1) == linear(f32=None, b16=FAKE, resid=FAKE) == linear(f32=None, b16=FAKE, sign=-1.0) == INVALID
    assert linear(bias=ODD) == linear(resid=ODD) == INVALID
    assert linear(sign=float("nan")) == linear(sign=float("inf")) == INVALID
    for M in (4, 100, 2048):
        need = w4.workspace_bytes(cfg, M)
        if need:
            assert linear(M=M, ws=None) == linear(M=M, ws=ODD) == linear(M=M, n=need - 1) == INVALID
    wide = ctypes.byref(_w4(N=1 << 20).c())
    assert L.lsh_linear_w4(wide, 1 << 11, FAKE, 0, FAKE, None, None, 1.0, 0, FAKE, None, FAKE, BIG, None) == UNSUPPORTED


@pytest.mark.parametrize("N", [1025, 1537, 50257, (1 << 22) - 15])
def test_w4_rows_up_to_their_limit_taken(built, N):
    """M N < 2^31, where N does not divide 2^31 too: the last M is turned away for the missing rows alone."""
    most = ((1 << 31) - 1) // N
    r = ctypes.byref(_w4(N=N, K=32).c())
    status = lambda M: w4.lib().lsh_linear_w4(r, M, None, 0, FAKE, None, None, 1.0, 0, FAKE, None, FAKE, BIG, None)
    assert most <= 1 << 21 and status(most) == INVALID and status(most + 1) == UNSUPPORTED


@pytest.mark.parametrize("N,K,taken", [(1 << 22, 8160, True), ((1 << 18) + 1, (1 << 17) - 32, True), (1 << 22, 8192, False),
                                       (1 << 18, 1 << 17, False), ((1 << 18) - 1, 1 << 17, True)])
def test_w4_matrices_up_to_their_limit_taken(built, N, K, taken):
    """N K < 2^35, whatever the rest of the last tiles."""
    assert (N * K < 1 << 35) == taken
    for kind in (dict(group=32, zeros=True), dict(type="e2m1", group=32)):
        assert (w4.weight_bytes(_w4(N=N, K=K, **kind)) > N * K // 2) == taken


def test_sizes_past_32_bits_refused(built):
    """The C structures hold 32 bits: 2^32 + 64 would pass as 64."""
    for bad in (dict(N=(1 << 32) + 64), dict(K=(1 << 32) + 64), dict(group=(1 << 32) + 32), dict(N=-1)):
        with pytest.raises(ValueError, match="out of range"):
            w4.weight_bytes(_w4(**bad))
    with pytest.raises(ValueError, match="out of range"):
        residual.workspace_bytes(_res(D=(1 << 32) + 64))


def test_linear_without_weights_refused(built):
    with pytest.raises(ValueError, match="packed"):
        w4.lsh_linear_w4(_w4(), torch.zeros(1, 256, dtype=torch.bfloat16), None)
    with pytest.raises(ValueError, match="sign"):
        w4.lsh_linear_w4(_w4(), torch.zeros(1, 256, dtype=torch.bfloat16), torch.zeros(8), sign=-1.0, dtype=torch.bfloat16)


@pytest.mark.parametrize("N,K,M", [(4096, 4096, 700), (1000, 8224, 2100), (8192, 8192, 2049), (16, 32, 300)])
def test_w4_workspace_of_up_to(built, N, K, M):
    cfg = _w4(N=N, K=K)
    assert w4.workspace(cfg, M, "cpu").numel() >= max(w4.workspace_bytes(cfg, m) for m in range(1, M + 1))


def test_w4_sizes(built):
    """A quarter of bf16's bytes, the scales' and the tiles' rest."""
    assert w4.weight_bytes(_w4(N=4096, K=1024)) == 4096 * 1024 // 2 + 4096 * 8 * 2
    assert w4.weight_bytes(_w4(N=4096, K=1024, group=32, zeros=True)) == 4096 * 1024 // 2 + 4096 * 32 * 3
    assert w4.weight_bytes(_w4(N=4096, K=1024, type="e2m1", group=32)) == 4096 * 1024 // 2 + 4096 * 32
    assert w4.weight_bytes(_w4(N=1, K=32)) == 1024 + 256


# ----------------------------------------------------------------------------
# the step between two blocks


def _res(**kw):
    base = dict(T=6, D=64, norm="layer", gate="sigmoid")
    base.update(kw)
    return residual.ResidualConfig(**base)


BAD_RES = [(dict(T=0), INVALID), (dict(D=0), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID),
           (dict(alpha=float("inf")), INVALID), (dict(f_stride=56), INVALID), (dict(f_stride=68), INVALID),
           (dict(gate_stride=-64), INVALID), (dict(D=60), UNSUPPORTED), (dict(D=8200), UNSUPPORTED),
           (dict(T=1 << 31), UNSUPPORTED), (dict(gate_stride=1 << 32), UNSUPPORTED)]
WEIGHTS = residual.ResidualWeightsC(*[0x1000] * 5)
GRADS = residual.ResidualGradsC(*[0x1000] * 8)


def _fwd(c, dtype=1, x=FAKE, f=FAKE, gate=FAKE, w=WEIGHTS, y=FAKE, z=FAKE):
    return residual.lib().lsh_residual_norm_fwd(ctypes.byref(c) if c is not None else None, dtype, x, f, gate,
                                                ctypes.byref(w) if w is not None else None, y, z, None)


def _bwd(c, dtype=1, y=FAKE, f=FAKE, gate=FAKE, w=WEIGHTS, dy=FAKE, dz=FAKE, g=GRADS, ws=FAKE, n=BIG):
    return residual.lib().lsh_residual_norm_bwd(ctypes.byref(c) if c is not None else None, dtype, y, f, gate,
                                                ctypes.byref(w) if w is not None else None, dy, dz,
                                                ctypes.byref(g) if g is not None else None, ws, n, None)


@pytest.mark.parametrize("bad,status", BAD_RES)
def test_residual_config_refused(built, bad, status):
    cfg = _res(**bad)
    assert residual.workspace_bytes(cfg) == 0
    assert _fwd(cfg.c()) == _bwd(cfg.c()) == status


def _with(base, **kw):
    c = type(base).from_buffer_copy(base)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def test_residual_arguments_refused(built):
    c = _res().c()
    need = residual.workspace_bytes(_res())
    assert need > 0
    for field, bad in (("norm", 2), ("norm", -1), ("gate", 3), ("gate", -1)):
        assert _fwd(_with(c, **{field: bad})) == _bwd(_with(c, **{field: bad})) == INVALID
    assert _fwd(None) == _bwd(None) == _fwd(c, w=None) == _bwd(c, w=None) == _bwd(c, g=None) == INVALID
    assert _fwd(c, dtype=4) == _bwd(c, dtype=4) == INVALID
    for p in (None, ODD):
        for name in ("gate", "y", "z"):
            assert _fwd(c, **{name: p}) == INVALID, name
        for name in ("gate", "y", "dz", "ws"):
            assert _bwd(c, **{name: p}) == INVALID, name
    for name in ("x", "f"):
        assert _fwd(c, **{name: ODD}) == INVALID
    assert _bwd(c, f=ODD) == _bwd(c, dy=ODD) == _bwd(c, n=need - 1) == INVALID
    # what goes without a branch, and what not
    none = _res(gate="none", post=False).c()
    rest = residual.ResidualWeightsC(0, 0, 0, 0x1000, 0)
    assert _fwd(c, f=None) == _fwd(none, x=None, f=None, gate=None, w=rest) == INVALID
    assert _fwd(none, f=None, gate=None, w=_with(rest, scale=0x1000)) == INVALID
    for name in ("post_g", "pre_g"):
        assert _fwd(c, w=_with(WEIGHTS, **{name: 0})) == _bwd(c, w=_with(WEIGHTS, **{name: 0})) == INVALID
        off = _res(**{name[:-2]: False}).c()
        assert _fwd(off, z=FAKE if name == "post_g" else None) == INVALID  # a gain without its norm
    assert _fwd(_res(gate="none").c()) == INVALID  # a gate without its kind
    for name in residual.WEIGHTS:
        assert _fwd(c, w=_with(WEIGHTS, **{name: 0x1008})) == INVALID
    for name in residual.GRADS:
        assert _bwd(c, g=_with(GRADS, **{name: 0})) == INVALID, name  # a gradient that the call has
        assert _bwd(c, g=_with(GRADS, **{name: 0x1008})) == INVALID, name
    for name in ("scale", "post_b", "pre_b"):  # and one that it has not
        assert _bwd(c, w=_with(WEIGHTS, **{name: 0})) == INVALID, name
    pre = _res(pre=False, post=False, gate="none").c()
    only = residual.ResidualWeightsC(0x1000, 0, 0, 0, 0)
    grads = residual.ResidualGradsC(0x1000, 0x1000, 0, 0x1000, 0, 0, 0, 0)
    assert _bwd(pre, gate=None, w=only, dy=None, dz=None, g=grads) == INVALID  # no gradient at all
    assert _bwd(pre, gate=None, w=only, g=grads) == INVALID  # dz without pre


# ----------------------------------------------------------------------------
# the cache's append


PAGES = cache.CachePagesC(*[0x1000] * 5)
SEQS = cache.CacheSeqsC(*[0x1000] * 3)


def _pair(shared=False, **kw):
    H, Hkv = (2, 2) if shared else (4, 2)
    c = cache.CacheConfig(n_seq=3, T=8, H=H, Hkv=Hkv, n_pages=10, max_pages=4, page=16, type="e4m3", shared_qk=shared)
    k = dict(T=8, Hq=H, Hk=0 if shared else Hkv)
    k.update(kw)
    return c, qk.QkConfig(**k)


def _append(c, k, dtype=1, pages=PAGES, seqs=SEQS, args=(FAKE, FAKE, FAKE, FAKE, FAKE)):
    ref = lambda s: None if s is None else ctypes.byref(s)
    return cache.lib().lsh_cache_append(ref(c), ref(k), dtype, ref(pages), ref(seqs), *args, None)


@pytest.mark.parametrize("bad,status", [
    (dict(T=9), INVALID), (dict(L=8), INVALID), (dict(Hq=3), INVALID), (dict(Hk=4), INVALID), (dict(Hk=0), INVALID),
    (dict(d=32), INVALID), (dict(rot=66), INVALID), (dict(rot=-16), INVALID), (dict(rot=7), INVALID),
    (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(x_stride=504), INVALID), (dict(x_stride=514), INVALID),
    (dict(rot=8), UNSUPPORTED), (dict(x_stride=1 << 40), UNSUPPORTED)])
def test_append_config_refused(built, bad, status):
    c, k = _pair(**bad)
    assert _append(c.c(), k.c()) == status


def test_append_arguments_refused(built):
    c, k = (x.c() for x in _pair())
    assert _append(None, k) == _append(c, None) == _append(c, k, pages=None) == _append(c, k, seqs=None) == INVALID
    assert _append(c, k, dtype=9) == INVALID
    for i in range(5):  # x, gain_q, gain_k, freq, q
        for p in (None, ODD):
            if i == 3 and p is ODD:
                continue  # freq needs no alignment
            assert _append(c, k, args=[p if j == i else FAKE for j in range(5)]) == INVALID, i
    shared = [x.c() for x in _pair(shared=True)]
    assert _append(*shared) == INVALID  # a key gain that no head has
    assert _append(*shared, pages=cache.CachePagesC(0x1000, 0x1000, 0x1000, 0x1000, 0), args=(FAKE, FAKE, None, FAKE, FAKE)) == INVALID
    big = cache.CacheConfig(n_seq=1, T=1 << 28, H=1, Hkv=1, n_pages=4, max_pages=4, page=16, type="bf16").c()
    assert _append(big, qk.QkConfig(T=1 << 28, Hq=1).c(), args=(FAKE, FAKE, None, FAKE, FAKE)) == UNSUPPORTED


# ----------------------------------------------------------------------------
# the bindings


class OnGpu(torch.Tensor):
    """A CPU tensor that passes for a GPU one, as its views do."""
    is_cuda = property(lambda self: True)


def on_gpu(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


BF = torch.bfloat16


@pytest.fixture
def no_library(monkeypatch):
    def refuse():
        raise AssertionError("the library was reached")
    for m in (cache, w4, residual):
        monkeypatch.setattr(m, "lib", refuse)
    monkeypatch.setattr(w4, "weight_bytes", lambda cfg: 1 << 20)
    monkeypatch.setattr(w4, "workspace_bytes", lambda cfg, M: 0)
    monkeypatch.setattr(residual, "workspace_bytes", lambda cfg: 256)


def test_w4_binding_refuses(no_library):
    cfg = _w4(N=16, K=64)
    packed = on_gpu(1 << 20, dtype=torch.uint8)
    a = on_gpu(3, 64, dtype=BF)
    bad = [
        (ValueError, "GPU", lambda: w4.lsh_linear_w4(cfg, torch.zeros(3, 64, dtype=BF), packed)),
        (ValueError, "shape", lambda: w4.lsh_linear_w4(cfg, on_gpu(3, 32, dtype=BF), packed)),
        (ValueError, "shape", lambda: w4.lsh_linear_w4(cfg, on_gpu(0, 64, dtype=BF), packed)),
        (ValueError, "dtype", lambda: w4.lsh_linear_w4(cfg, on_gpu(3, 64), packed)),
        (ValueError, "stride", lambda: w4.lsh_linear_w4(cfg, on_gpu(1, 64, dtype=BF).expand(3, 64), packed)),
        (ValueError, "contiguous", lambda: w4.lsh_linear_w4(cfg, on_gpu(64, 3, dtype=BF).t(), packed)),
        (ValueError, "packed", lambda: w4.lsh_linear_w4(cfg, a, packed[:100])),
        (ValueError, "packed", lambda: w4.lsh_linear_w4(cfg, a, on_gpu(1 << 20))),
        (ValueError, "bias", lambda: w4.lsh_linear_w4(cfg, a, packed, bias=on_gpu(15))),
        (ValueError, "resid", lambda: w4.lsh_linear_w4(cfg, a, packed, resid=on_gpu(3, 16, dtype=BF))),
        (TypeError, "dtype", lambda: w4.lsh_linear_w4(cfg, a, packed, dtype=torch.float16)),
        (ValueError, "out", lambda: w4.lsh_linear_w4(cfg, a, packed, out=on_gpu(3, 17))),
        (ValueError, "workspace", lambda: w4.lsh_linear_w4(cfg, a, packed, workspace=torch.zeros(256, dtype=torch.uint8))),
        (ValueError, "w", lambda: w4.lsh_w4_quantize(cfg, on_gpu(16, 63))),
        (TypeError, "dtype", lambda: w4.lsh_w4_quantize(cfg, on_gpu(16, 64, dtype=torch.float16))),
        (ValueError, "codes", lambda: w4.lsh_w4_pack(cfg, on_gpu(16, 64, dtype=torch.uint8), on_gpu(16, 1, dtype=BF))),
        (ValueError, "scales", lambda: w4.lsh_w4_pack(cfg, on_gpu(16, 32, dtype=torch.uint8), on_gpu(16, 1))),
        (ValueError, "zeros", lambda: w4.lsh_w4_pack(cfg, on_gpu(16, 32, dtype=torch.uint8), on_gpu(16, 1, dtype=BF),
                                                     on_gpu(16, 1, dtype=torch.uint8))),
    ]
    for error, match, call in bad:
        with pytest.raises(error, match=match):
            call()


def test_residual_binding_refuses(no_library):
    cfg, D = _res(), 64
    vec = lambda: on_gpu(D)
    w = residual.ResidualWeights(post_g=vec(), pre_g=vec())
    x, f = on_gpu(6, D), on_gpu(6, D, dtype=BF)
    fwd, bwd = residual.lsh_residual_norm_fwd, residual.lsh_residual_norm_bwd
    bad = [
        ("x is required", lambda: fwd(cfg, None, None, None, w)),
        ("without f", lambda: fwd(cfg, x, None, f, w)),
        ("gate", lambda: fwd(cfg, x, f, None, w)),
        ("gate", lambda: fwd(cfg, x, f, x, w)),  # of another dtype
        ("GPU", lambda: fwd(cfg, x, torch.zeros(6, D, dtype=BF), f, w)),
        ("shape", lambda: fwd(cfg, x, on_gpu(5, D, dtype=BF), f, w)),
        ("stride", lambda: fwd(cfg, x, on_gpu(1, D, dtype=BF).expand(6, D), f, w)),
        ("contiguous", lambda: fwd(cfg, x, on_gpu(D, 6, dtype=BF).t(), f, w)),
        ("x", lambda: fwd(cfg, on_gpu(6, D, dtype=BF), f, f, w)),
        ("z goes", lambda: fwd(_res(pre=False), x, f, f, residual.ResidualWeights(post_g=vec()), z=f)),
        ("post_g is required", lambda: fwd(cfg, x, f, f, residual.ResidualWeights(pre_g=vec()))),
        ("go with pre", lambda: fwd(_res(pre=False), x, f, f, w)),
        ("pre_b", lambda: fwd(cfg, x, f, f, residual.ResidualWeights(post_g=vec(), pre_g=vec(), pre_b=on_gpu(63)))),
        ("dtype", lambda: fwd(cfg, x, f, f, w, dtype=torch.float32)),
        ("dz", lambda: bwd(cfg, x, f, f, w, x, None)),
        ("y is required", lambda: bwd(cfg, None, f, f, w, x, x)),
        ("dy", lambda: bwd(cfg, x, f, f, w, on_gpu(6, 32), x)),
        ("grads", lambda: bwd(cfg, x, f, f, w, x, x, grads={"dscale": vec()})),
        ("grads", lambda: bwd(cfg, x, f, f, w, x, x, grads={"dgain": vec()})),
        ("workspace", lambda: bwd(cfg, x, f, f, w, x, x, workspace=torch.zeros(256, dtype=torch.uint8))),
    ]
    for match, call in bad:
        with pytest.raises(ValueError, match=match):
            call()


def test_append_binding_refuses(no_library):
    c, k = _pair()
    p = cache.Pages.empty(c, "cpu")
    p = cache.Pages(*(t.as_subclass(OnGpu) for t in (p.k, p.v, p.k_scale, p.v_scale)))
    s = cache.Sequences(*(on_gpu(*shape, dtype=torch.int32) for shape in ((4,), (3,), (3, 4))))
    x, g, fr = on_gpu(8, 8 * 64), on_gpu(64), on_gpu(32)
    call = lambda k=k, x=x, gq=g, gk=g, fr=fr, **kw: cache.lsh_cache_append(c, k, p, s, x, gq, gk, fr, **kw)
    bad = [
        ("expected", lambda: call(k=_pair(Hk=0)[1])), ("expected", lambda: call(k=_pair(L=4)[1])),
        ("shape", lambda: call(x=on_gpu(8, 7 * 64))), ("stride", lambda: call(x=on_gpu(1, 8 * 64).expand(8, 8 * 64))),
        ("GPU", lambda: call(x=torch.zeros(8, 8 * 64))), ("gain_k", lambda: call(gk=None)), ("gain_k", lambda: call(gq=None)),
        ("gain_q", lambda: call(gq=on_gpu(4, 64))), ("freq", lambda: call(fr=on_gpu(16))),
        ("q has dtype", lambda: call(q=on_gpu(8, 4, 64))), ("stride", lambda: call(q=on_gpu(1, 4, 64, dtype=BF).expand(8, 4, 64))),
    ]
    for match, f in bad:
        with pytest.raises(ValueError, match=match):
            f()


@pytest.mark.parametrize("make", [_w4, _res])
def test_configurations_copy_and_compare(built, make):
    used = make()
    used.ref()
    assert used == make() and hash(used) == hash(make())
    assert pickle.loads(pickle.dumps(used)) == used and copy.deepcopy(used) == used
    with pytest.raises(KeyError):
        (w4.W4Config(1, 32, type="int8") if make is _w4 else _res(norm="batch")).c()
