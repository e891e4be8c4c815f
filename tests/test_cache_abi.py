"""The cache's and the per-head norm's C ABI and binding without a GPU: exported symbols, workspaces, and
every refusal before any HIP call."""
import ctypes
import os
import re

import pytest
import torch

from paper_2001_04451_amd import cache, lsh, qk

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = ctypes.c_void_p(0x1000)  # never dereferenced: every call below fails validation
ODD = ctypes.c_void_p(0x1008)
INVALID, UNSUPPORTED = lsh.LSH_ERR_INVALID, lsh.LSH_ERR_UNSUPPORTED
BIG = 1 << 40


@pytest.fixture(scope="module")
def built():
    if not os.path.exists(lsh.LIB_PATH):
        pytest.skip("liblsh.so not built (run __graft_entry__.build())")


@pytest.mark.parametrize("module,header", [(qk, "lsh_qk.h"), (cache, "lsh_cache.h")])
def test_header_symbols_exported(built, module, header):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
    assert set(re.findall(r"\b(lsh_[a-z0-9_]+)\s*\(", text)) == set(module.EXPORTED)
    for name in module.EXPORTED:
        assert hasattr(module.lib(), name)


def _qk(**kw):
    base = dict(T=6, Hq=2, Hk=1, L=3)
    base.update(kw)
    return qk.QkConfig(**base)


BAD_QK = [(dict(T=0), INVALID), (dict(Hq=0), INVALID), (dict(Hk=-1), INVALID), (dict(L=4), INVALID),
          (dict(L=-3), INVALID), (dict(rot=66), INVALID), (dict(rot=-2), INVALID), (dict(rot=31), INVALID),
          (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(d=0), INVALID),
          (dict(x_stride=100), INVALID), (dict(x_stride=201), INVALID), (dict(dx_stride=194), INVALID),
          (dict(rot=24), UNSUPPORTED), (dict(d=128), UNSUPPORTED), (dict(Hq=1024), UNSUPPORTED),
          (dict(T=1 << 30, L=0), UNSUPPORTED), (dict(x_stride=1 << 40), UNSUPPORTED)]


@pytest.mark.parametrize("bad,status", BAD_QK)
def test_qk_config_refused(built, bad, status):
    L, c = qk.lib(), _qk(**bad).c()
    assert qk.qk_workspace_bytes(_qk(**bad)) == 0
    assert L.lsh_qk_norm_rotate_fwd(ctypes.byref(c), 1, *[FAKE] * 7, None) == status
    assert L.lsh_qk_norm_rotate_bwd(ctypes.byref(c), 1, *[FAKE] * 11, BIG, None) == status


def test_qk_pointers_refused(built):
    L, c = qk.lib(), _qk().c()
    need = qk.qk_workspace_bytes(_qk())
    assert need >= 2 * 64 * 4
    fwd = lambda args, dt=1: L.lsh_qk_norm_rotate_fwd(ctypes.byref(c), dt, *args, None)
    bwd = lambda args, n=need, dt=1: L.lsh_qk_norm_rotate_bwd(ctypes.byref(c), dt, *args, n, None)
    assert L.lsh_qk_norm_rotate_fwd(None, 1, *[FAKE] * 7, None) == INVALID
    assert L.lsh_qk_norm_rotate_bwd(None, 1, *[FAKE] * 11, need, None) == INVALID
    assert fwd([FAKE] * 7, 7) == INVALID and bwd([FAKE] * 11, dt=7) == INVALID
    for i in range(7):  # x, gain_q, gain_k, freq, pos, q, k
        for p in (None, ODD):
            if i in (3, 4) and p is ODD or i == 4:
                continue  # freq needs no alignment; pos may be NULL
            assert fwd([p if j == i else FAKE for j in range(7)]) == INVALID, i
    for i in range(11):  # x, gain_q, gain_k, freq, pos, dq, dk, dx, dgain_q, dgain_k, workspace
        for p in (None, ODD):
            if i == 4 or (p is ODD and i in (3, 8, 9)):
                continue
            assert bwd([p if j == i else FAKE for j in range(11)]) == INVALID, i
    assert bwd([FAKE] * 11, need - 1) == INVALID


def _cache(**kw):
    base = dict(n_seq=3, T=8, H=4, Hkv=2, n_pages=10, max_pages=4, page=16, type="e4m3", shared_qk=False)
    base.update(kw)
    return cache.CacheConfig(**base)


BAD_CACHE = [(dict(T=0), INVALID), (dict(n_seq=0), INVALID), (dict(H=0), INVALID), (dict(Hkv=0), INVALID),
             (dict(H=3), INVALID), (dict(shared_qk=True), INVALID), (dict(page=0), INVALID),
             (dict(n_pages=0), INVALID), (dict(max_pages=0), INVALID), (dict(max_new=-1), INVALID),
             (dict(scale=float("inf")), INVALID), (dict(self_mask=float("nan")), INVALID), (dict(d=0, scale=1.0), INVALID),
             (dict(q_stride=128), INVALID), (dict(k_stride=132), INVALID), (dict(v_stride=64), INVALID),
             (dict(d=128), UNSUPPORTED), (dict(page=8), UNSUPPORTED), (dict(page=48), UNSUPPORTED),
             (dict(page=8192), UNSUPPORTED), (dict(max_pages=1 << 27), UNSUPPORTED), (dict(H=2048), UNSUPPORTED),
             (dict(n_seq=(1 << 14) + 1), UNSUPPORTED), (dict(T=1 << 30), UNSUPPORTED), (dict(q_stride=1 << 40), UNSUPPORTED)]


def _calls(c, pages, seqs, n=BIG, dtype=1):
    L = cache.lib()
    head = (ctypes.byref(c) if c is not None else None, dtype, ctypes.byref(pages), ctypes.byref(seqs))
    return (L.lsh_cache_write(*head, FAKE, FAKE, None), L.lsh_cache_read(*head, FAKE, FAKE, None),
            L.lsh_cache_attn_fwd(*head, FAKE, FAKE, FAKE, FAKE, n, None))


PAGES = cache.CachePagesC(*[0x1000] * 5)
SEQS = cache.CacheSeqsC(*[0x1000] * 3)


@pytest.mark.parametrize("bad,status", BAD_CACHE)
def test_cache_config_refused(built, bad, status):
    assert cache.workspace_bytes(_cache(**bad)) == 0
    assert set(_calls(_cache(**bad).c(), PAGES, SEQS)) == {status}


def test_cache_types_and_pointers_refused(built):
    L, cfg = cache.lib(), _cache()
    c = cfg.c()
    c.type = 3
    assert set(_calls(c, PAGES, SEQS)) == {INVALID}
    c.type = -1
    assert set(_calls(c, PAGES, SEQS)) == {INVALID}
    c = cfg.c()
    assert set(_calls(None, PAGES, SEQS)) == {INVALID}
    assert set(_calls(c, PAGES, SEQS, dtype=5)) == {INVALID}
    for i, name in enumerate(("k", "v", "k_scale", "v_scale")):
        for p in (0, 0x1008):
            pages = cache.CachePagesC(*[0x1000] * 5)
            setattr(pages, name, p)
            assert set(_calls(c, pages, SEQS)) == {INVALID}, name
    for name in ("first", "length", "table"):
        seqs = cache.CacheSeqsC(*[0x1000] * 3)
        setattr(seqs, name, 0)
        assert set(_calls(c, PAGES, seqs)) == {INVALID}, name
    shared = _cache(H=2, shared_qk=True).c()
    assert set(_calls(shared, cache.CachePagesC(0x1000, 0x1000, 0x1000, 0x1000, 0), SEQS)) == {INVALID}
    head = (ctypes.byref(c), 1, ctypes.byref(PAGES), ctypes.byref(SEQS))
    for args in ((None, FAKE), (FAKE, None), (ODD, FAKE), (FAKE, ODD)):
        assert L.lsh_cache_write(*head, *args, None) == INVALID
    for args in ((None, None), (ODD, None), (None, ODD)):
        assert L.lsh_cache_read(*head, *args, None) == INVALID
    need = cache.workspace_bytes(cfg)
    for i in (0, 1, 3):  # q, out, workspace
        for p in (None, ODD):
            args = [p if j == i else FAKE for j in range(4)]
            assert L.lsh_cache_attn_fwd(*head, *args, need, None) == INVALID, i
    assert L.lsh_cache_attn_fwd(*head, *[FAKE] * 4, need - 1, None) == INVALID
    # fp32 queries, and a self mask too small to be exact
    assert L.lsh_cache_attn_fwd(ctypes.byref(c), 0, *head[2:], *[FAKE] * 4, need, None) == UNSUPPORTED
    weak = _cache(H=2, shared_qk=True, self_mask=100.0).c()
    assert L.lsh_cache_attn_fwd(ctypes.byref(weak), 1, *head[2:], *[FAKE] * 4, BIG, None) == UNSUPPORTED


def test_binding_refuses_before_the_library():
    """Shapes, dtypes and devices, on CPU tensors."""
    cfg = _cache()
    pages = cache.Pages.empty(cfg, "cpu")
    seqs = cache.Sequences(*(torch.zeros(s, dtype=torch.int32) for s in (4, 3, (3, 4))))
    rows = torch.zeros(8, 2, 64)
    with pytest.raises(ValueError, match="GPU"):
        cache.lsh_cache_write(cfg, pages, seqs, rows, rows)
    with pytest.raises(ValueError, match="GPU"):
        qk.lsh_qk_norm_rotate_fwd(_qk(), torch.zeros(6, 192), torch.ones(64), torch.ones(64), torch.ones(32))
    with pytest.raises(KeyError):
        _cache(type="int8").c()


def test_configurations_copy_and_compare(built):
    """A configuration that has been used compares, copies and pickles as one that has not, and c() is the caller's own."""
    import copy
    import pickle
    for make in (_cache, _qk):
        used = make()
        used.ref()
        assert used == make() and hash(used) == hash(make())
        assert pickle.loads(pickle.dumps(used)) == used and copy.deepcopy(used) == used
        used.c().T = 99
        assert used.c().T == make().T
