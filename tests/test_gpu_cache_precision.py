"""Attention of a few tokens over the cache: weights carry 16 bits there, also
beside values that are not finite (one MI355X)."""
import numpy as np
import pytest
import torch

from oracle import cache as C
from paper_2001_04451_amd import cache

from gpu_common import log
from test_gpu_cache import Case, gpu  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shared", [True, False])
@pytest.mark.parametrize("type_", ["bf16", "e4m3", "e2m1"])
def test_weights_of_few_tokens_keep_sixteen_bits(gpu, type_, shared):  # noqa: F811
    """A weight is off by 2^-16 of it at most (what its bf16 rounding leaves, itself at most 2^-8 of it, is rounded to
    bf16 once more); the sums of up to 700 keys take fewer than 700 roundings of 2^-24 to fp32.  Products, sum and
    division together: (2^-16 + 700 2^-24) twice, below 2^-12, and the output's own rounding of 2^-8."""
    c = Case(type_, shared, 8 if not shared else 4, 4, 32, [1, 60, 333, 700], [1, 2, 1, 3], seed=21)
    host, kr, vr = c.host_pages()
    log("cache attention precision", type_, shared)
    out, _ = cache.lsh_cache_attn_fwd(c.cfg, c.pages(host, gpu), c.seqs(gpu), c.q.to(gpu))
    inv = None if host[4] is None else host[4].astype(np.float64)
    ref, _, spread, _ = C.attend(c.q.double().numpy(), kr, vr, inv, c.first, c.lens, c.table, c.page, 0.125, c.shared,
                                 c.cfg.self_mask)
    # logits: sums of 64 products of up to |q||k|/8 (below 64 in all) in fp32, 70 roundings, and twice for numerator and sum
    dz = 2 * 70 * 2.0 ** -24 * 64 * np.log(2)
    tol = (2.0 ** -12 + dz) * spread + 2.0 ** -8 * np.abs(ref)
    longest = 1 if shared else np.linalg.norm(kr, axis=-1).max()
    assert (np.linalg.norm(c.q.double().numpy(), axis=-1) * 0.125 * longest < 64).all()
    assert (np.abs(out.double().cpu().numpy() - ref) <= tol).all()


@pytest.mark.parametrize("shared", [True, False])
def test_infinite_values_of_seen_keys(gpu, shared):  # noqa: F811
    """An infinite value that a row sees makes its output infinite, two of different sign NaN; the other dimensions and
    rows are as without it."""
    def run(odd):
        c = Case("bf16", shared, 8 if not shared else 4, 4, 16, [900, 70], [1, 1], seed=5)
        if odd:
            for s, p, d, x in ((0, 3, 5, np.inf), (0, 470, 9, -np.inf), (0, 40, 20, np.inf), (0, 600, 20, -np.inf),
                               (1, 31, 63, np.inf)):
                c.v[c.table[s, p // 16], 1, p % 16, d] = x
        host, _, _ = c.host_pages()
        return cache.lsh_cache_attn_fwd(c.cfg, c.pages(host, gpu), c.seqs(gpu), c.q.to(gpu))

    log("cache attention infinite values", shared)
    (out, lse), (want, want_lse) = run(True), run(False)
    G = 1 if shared else 2
    want = want.clone()
    mine = slice(G, 2 * G)  # the query heads of key head 1
    want[0, mine, 5], want[0, mine, 9], want[0, mine, 20], want[1, mine, 63] = np.inf, -np.inf, np.nan, np.inf
    assert torch.equal(lse, want_lse)
    torch.testing.assert_close(out, want, rtol=0, atol=0, equal_nan=True)


@pytest.mark.parametrize("shared", [True, False])
@pytest.mark.parametrize("type_", ["bf16", "e4m3", "e2m1"])
def test_weights_of_short_chunks_keep_sixteen_bits(gpu, type_, shared):  # noqa: F811
    """As for few tokens, and infinite values of keys that all rows of a tile see, or some."""
    c = Case(type_, shared, 4, 4 if shared else 2, 32, [300, 700], [70, 40], seed=22)
    host, kr, vr = c.host_pages()
    log("cache attention precision of chunks", type_, shared)
    out, _ = cache.lsh_cache_attn_fwd(c.cfg, c.pages(host, gpu), c.seqs(gpu), c.q.to(gpu))
    inv = None if host[4] is None else host[4].astype(np.float64)
    ref, _, spread, _ = C.attend(c.q.double().numpy(), kr, vr, inv, c.first, c.lens, c.table, c.page, 0.125, c.shared,
                                 c.cfg.self_mask)
    dz = 2 * 70 * 2.0 ** -24 * 64 * np.log(2)
    tol = (2.0 ** -12 + dz) * spread + 2.0 ** -8 * np.abs(ref)
    assert (np.abs(out.double().cpu().numpy() - ref) <= tol).all()
    if type_ != "bf16":
        return
    for s, p, d, x in ((0, 100, 5, np.inf), (0, 250, 9, -np.inf), (1, 3, 11, np.inf), (1, 500, 11, -np.inf)):
        c.v[c.table[s, p // 32], 1, p % 32, d] = x
    host, _, _ = c.host_pages()
    odd, _ = cache.lsh_cache_attn_fwd(c.cfg, c.pages(host, gpu), c.seqs(gpu), c.q.to(gpu))
    want, G = out.clone(), c.H // c.Hkv
    mine = slice(G, 2 * G)
    want[:70, mine, 5], want[70:, mine, 11] = np.inf, np.nan
    n = 250 - 230 + (1 if shared else 0)  # new tokens that do not see position 250
    want[n:70, mine, 9] = -np.inf
    torch.testing.assert_close(odd, want, rtol=0, atol=0, equal_nan=True)
