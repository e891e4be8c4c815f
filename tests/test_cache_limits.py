"""Sizes at the ends of what the norm's, the cache's and its attention's entry points take, on the CPU: no call below is
launched."""
import ctypes
import random

from paper_2001_04451_amd import cache, qk

from test_cache_abi import BIG, FAKE, INVALID, PAGES, SEQS, UNSUPPORTED, _cache, built  # noqa: F401


def test_grids_past_the_launch_limit_refused(built):  # noqa: F811
    """HIP launches fewer than 2^32 threads a dimension: calls that would need more are refused before any launch, those
    right below are not (they go on to the missing pointer)."""
    Q, L = qk.lib(), cache.lib()
    for T, status in ((2 ** 28 - 16, INVALID), (2 ** 28 - 15, UNSUPPORTED), (2 ** 30, UNSUPPORTED)):
        cfg = qk.QkConfig(T=T, Hq=1)
        assert Q.lsh_qk_norm_rotate_fwd(ctypes.byref(cfg.c()), 1, None, *[FAKE] * 6, None) == status
        assert (qk.qk_workspace_bytes(cfg) > 0) == (status == INVALID)
    rows = lambda T, Hkv: _cache(T=T, H=Hkv, Hkv=Hkv).c()
    # eight tokens and four rows (k and v of two heads) a wave, four waves a workgroup of 256
    for T, Hkv, status in ((8 * (2 ** 26 - 4), 2, INVALID), (8 * (2 ** 26 - 4) + 1, 2, UNSUPPORTED),
                           (8 * (2 ** 26 - 4) + 1, 1, UNSUPPORTED), (2 ** 28, 1, INVALID), (2 ** 18, 1024, INVALID),
                           (2 ** 21 - 1, 1023, UNSUPPORTED)):
        head = (ctypes.byref(rows(T, Hkv)), 1, ctypes.byref(PAGES), ctypes.byref(SEQS))
        assert L.lsh_cache_write(*head, None, FAKE, None) == status, (T, Hkv)
        assert L.lsh_cache_read(*head, None, None, None) == status, (T, Hkv)
    # a workgroup for every 16 rows, for every sequence and head, and 16 lanes a row to join parts
    for kw, status in ((dict(T=2 ** 27, H=1, Hkv=1), INVALID), (dict(T=2 ** 29, H=1, Hkv=1, max_new=1), UNSUPPORTED),
                       (dict(T=2 ** 29, H=1, Hkv=1, n_seq=1, page=4096), INVALID),  # one prompt, 256 rows a workgroup
                       (dict(T=2 ** 14, H=1024, Hkv=1024, n_seq=2 ** 14, max_new=1), UNSUPPORTED),
                       (dict(T=2 ** 11, H=1024, Hkv=1024, n_seq=2 ** 11, max_new=1), INVALID)):
        cfg = _cache(**kw)
        head = (ctypes.byref(cfg.c()), 1, ctypes.byref(PAGES), ctypes.byref(SEQS))
        assert L.lsh_cache_attn_fwd(*head, None, FAKE, FAKE, FAKE, BIG, None) == status, kw
        assert (cache.workspace_bytes(cfg) > 0) == (status == INVALID), kw


def test_documented_sizes_are_taken(built):  # noqa: F811
    """T * H up to 2^27 and n_seq * Hkv up to 2^21 (and rows to write and read up to 2^28) never pass the launch limit."""
    rng = random.Random(1)
    L = cache.lib()
    size = lambda most: min(most, int(2 ** rng.uniform(0, most.bit_length())))
    for i in range(4000):
        Hkv = size(1024)
        H = Hkv * size(1024 // Hkv)
        n_seq = min(2 ** 14, 2 ** 21 // Hkv if i % 3 == 0 else size(2 ** 21 // Hkv))
        T = 2 ** 27 // H if i % 2 == 0 else size(2 ** 27 // H)
        page = 2 ** rng.randint(4, 12)
        cfg = _cache(T=T, H=H, Hkv=Hkv, n_seq=n_seq, page=page, max_pages=size(2 ** 30 // page), n_pages=8,
                     max_new=rng.choice([0, 1, 16, 17, size(2 ** 20)]))
        assert cache.workspace_bytes(cfg) > 0, cfg
        head = (ctypes.byref(_cache(T=2 * T, H=H, Hkv=Hkv, n_seq=n_seq).c()), 1, ctypes.byref(PAGES), ctypes.byref(SEQS))
        if 2 * T * Hkv <= 2 ** 28:
            assert L.lsh_cache_write(*head, None, FAKE, None) == INVALID, cfg
