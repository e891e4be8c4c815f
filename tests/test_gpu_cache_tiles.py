"""Every kernel of the attention over the cache against the fp64 oracle (one MI355X).

The kernels of large calls (64 rows a tile with weights as one bf16 number, 128 and 256 rows, 4-bit decoding with one
number) are chosen by the table's width and by max_new, which says only how many new tokens to expect: a wide table over
short sequences reaches them.  What the table holds behind a sequence's end counts for nothing."""
from dataclasses import replace

import numpy as np
import pytest
import torch

from oracle import cache as C
from paper_2001_04451_amd import cache

from gpu_common import log
from test_gpu_cache import TYPES, Case, check_attention, compare, gpu  # noqa: F401

pytestmark = pytest.mark.gpu

HEADS = {"shared2": (2, 2), "shared1": (1, 1), "group4": (8, 2), "group6": (6, 1)}
# rows a tile: rows of a sequence to expect, (query, key) pairs of the call by the table's width
TILES = {64: (64, 1 << 24), 128: (128, 1 << 24), 256: (256, 1 << 27)}


def widen(c, rows, pairs):
    """The case with a table so wide that T * H times its positions are at least `pairs`, and `rows` rows of a sequence
    expected."""
    G = c.H // c.Hkv
    max_new = max(1, rows // G)
    need = max(pairs, 2 * max_new * c.T * c.H)
    width = max(c.most, -(-need // (c.T * c.H * c.page)))
    more = c.rng.integers(-2, c.n_pages + 2, (len(c.lens), width - c.most)).astype(np.int32)
    c.table, c.most = np.concatenate([c.table, more], 1), width
    c.cfg = replace(c.cfg, max_pages=width, max_new=max_new)
    return c


def tiles(c, rows):
    return widen(c, *TILES[rows])


@pytest.mark.parametrize("shared", [True, False])
@pytest.mark.parametrize("type_", TYPES)
@pytest.mark.parametrize("rows", TILES)
def test_tiles_nothing_leaks_from_later_tokens(gpu, rows, type_, shared):  # noqa: F811
    """NaN and infinities in a new token's rows reach that token's successors alone, bit for bit."""
    def run(bad):
        c = Case(type_, shared, 2, 2, 16, [100, 420], [40, 290], seed=8)
        for s, p in bad.items():
            at = c.table[s, p // 16], p % 16
            c.v[at[0], 0, at[1], 5], c.v[at[0], 1, at[1], 40] = np.nan, np.inf
            c.k[at[0], :, at[1], 7] = np.inf if type_ == "bf16" else np.nan
        host, _, _ = c.host_pages()
        tiles(c, rows)
        return c, *cache.lsh_cache_attn_fwd(c.cfg, c.pages(host, gpu), c.seqs(gpu), c.q.to(gpu))

    bad = {0: 75, 1: 301}  # position of the bad row in each sequence
    log("cache tiles leaks", rows, type_, shared)
    (c, out, lse), (_, want, want_lse) = run(bad), run({})
    for s, p in bad.items():
        a, b = c.first[s], c.first[s + 1]
        n = p - (c.lens[s] - c.news[s]) + (1 if shared else 0)  # new tokens that do not see it
        assert torch.equal(out[a:a + n], want[a:a + n]) and torch.equal(lse[a:a + n], want_lse[a:a + n])
        assert torch.isnan(lse[a + n:b]).all() or torch.isnan(out[a + n:b].float()).any(-1).all()
