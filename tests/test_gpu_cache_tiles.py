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


# a whole prompt, a chunk, few tokens, one token, none; new tokens before position 0; one sequence alone
SHAPES = {
    "mixed": (16, [700, 40, 1, 129, 0, 350], [300, 1, 1, 17, 0, 350]),
    "beyond": (16, [3, 20, 90], [9, 25, 90]),
    "alone": (128, [900], [333]),
    "large pages": (4096, [4100, 77], [70, 77]),
}


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("type_", TYPES)
@pytest.mark.parametrize("rows", TILES)
def test_tiles(gpu, rows, type_, heads, shape):  # noqa: F811
    page, lens, news = SHAPES[shape]
    log("cache tiles", rows, type_, heads, shape)
    check_attention(tiles(Case(type_, heads.startswith("shared"), *HEADS[heads], page, lens, news, seed=len(shape),
                               fill="nan"), rows), gpu)


@pytest.mark.parametrize("scale", [0.01, 3.0, -0.125])
@pytest.mark.parametrize("rows", TILES)
def test_tiles_scales(gpu, rows, scale):  # noqa: F811
    """With 3.0 a running maximum is needed also with normalised keys."""
    for shared in (True, False):
        log("cache tiles scale", rows, scale, shared)
        check_attention(tiles(Case("bf16", shared, 2, 2, 16, [150, 400], [1, 170], scale=scale), rows), gpu)


@pytest.mark.parametrize("type_", TYPES)
@pytest.mark.parametrize("rows", TILES)
def test_tiles_bad_pages(gpu, rows, type_):  # noqa: F811
    """Holes in the first blocks and in the middle, and sequences without any page."""
    page, lens, news = SHAPES["mixed"]
    for shared in (True, False):
        c = Case(type_, shared, 2, 2, page, lens, news, seed=5, T=sum(news) + 3)
        c.table[0, 3], c.table[0, 21], c.table[3, 2] = -1, c.n_pages + 7, 2 ** 31 - 1
        c.table[5, 0], c.table[5, 1], c.table[5, 19] = -5, c.n_pages, -1
        log("cache tiles bad pages", rows, type_, shared)
        check_attention(tiles(c, rows), gpu)
        c = Case(type_, shared, 2, 2, page, lens, news, seed=6)
        c.table[:] = -1
        widen(c, *TILES[rows])
        out, lse, _ = check_attention(c, gpu)
        assert not out.any() and torch.isneginf(lse).all()


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


@pytest.mark.parametrize("shared", [True, False])
@pytest.mark.parametrize("rows", TILES)
def test_tiles_infinite_values_of_seen_keys(gpu, rows, shared):  # noqa: F811
    """Infinite values before the new tokens, which all of them see, and among them, which some see; the other dimensions
    and rows are as without them, bit for bit."""
    odd = ((0, 100, 5, np.inf), (0, 250, 9, -np.inf), (1, 3, 11, np.inf), (1, 500, 11, -np.inf), (1, 660, 63, np.inf))

    def run(odd):
        c = Case("bf16", shared, 4, 4 if shared else 2, 32, [300, 700], [70, 150], seed=22)
        for s, p, d, x in odd:
            c.v[c.table[s, p // 32], 1, p % 32, d] = x
        host, _, _ = c.host_pages()
        tiles(c, rows)
        return c, *cache.lsh_cache_attn_fwd(c.cfg, c.pages(host, gpu), c.seqs(gpu), c.q.to(gpu))

    log("cache tiles infinite values", rows, shared)
    (c, out, lse), (_, want, want_lse) = run(odd), run(())
    G = c.H // c.Hkv
    mine = slice(G, 2 * G)  # the query heads of key head 1
    want = want.clone()
    late = 1 if shared else 0
    want[:70, mine, 5], want[70:, mine, 11] = np.inf, np.nan
    want[250 - 230 + late:70, mine, 9] = -np.inf
    want[70 + 660 - 550 + late:, mine, 63] = np.inf
    assert torch.equal(lse, want_lse)
    torch.testing.assert_close(out, want, rtol=0, atol=0, equal_nan=True)


@pytest.mark.parametrize("rows", TILES)
def test_tiles_rows_outside_and_any_workspace(gpu, rows):  # noqa: F811
    """Sequences that neither begin at row 0 nor end at T; the same bits whatever the workspace holds, and nothing
    written beside it."""
    for shared in (True, False):
        c = Case("e4m3", shared, 4, 4 if shared else 2, 16, [700, 400, 3], [100, 290, 1], T=420)
        c.first += 5
        log("cache tiles rows outside", rows, shared)
        out, lse, (pages, seqs, q) = check_attention(tiles(c, rows), gpu)
        n = cache.workspace_bytes(c.cfg)
        for fill in (0, 255, 0x7F):
            ws = torch.full((n + 8192,), fill, dtype=torch.uint8, device=gpu)
            ws[:4096], ws[-4096:] = 0xA5, 0xA5
            out2, lse2 = torch.full_like(out, 7.0), torch.full_like(lse, 7.0)
            cache.lsh_cache_attn_fwd(c.cfg, pages, seqs, q, out=out2, lse=lse2, workspace=ws[4096:-4096])
            assert torch.equal(out, out2) and torch.equal(lse, lse2)
            assert (ws[:4096] == 0xA5).all() and (ws[-4096:] == 0xA5).all()


@pytest.mark.parametrize("rows", TILES)
def test_tiles_captured(gpu, rows):  # noqa: F811
    """A captured call replayed on other queries, lengths and splits of its rows among the sequences, against eager
    calls and the oracle."""
    cases = [tiles(Case("e4m3", True, 2, 2, 16, lens, news, seed=i), rows) for i, (lens, news) in
             enumerate((([500, 40, 7], [300, 1, 1]), ([1, 900, 64], [1, 237, 64]), ([260, 30, 12], [260, 30, 12])))]
    T, n_pages = cases[0].T, max(c.n_pages for c in cases)
    assert all(c.T == T and c.most == cases[0].most for c in cases)
    cfg = replace(cases[0].cfg, n_pages=n_pages)
    pages = cache.Pages.empty(cfg, gpu)
    parts = lambda p: (p.k, p.v, p.k_scale, p.v_scale, p.k_inv)
    for t in parts(pages):
        t.zero_()
    seqs, q = cases[0].seqs(gpu), torch.zeros(T, 2, 64, dtype=torch.bfloat16, device=gpu)
    out, lse, ws = torch.empty_like(q), torch.empty(T, 2, device=gpu), cache.workspace(cfg, gpu)
    log("cache tiles captured", rows)
    cache.lsh_cache_attn_fwd(cfg, pages, seqs, q, out=out, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cache.lsh_cache_attn_fwd(cfg, pages, seqs, q, out=out, lse=lse, workspace=ws)
    for c in cases * 2:
        host, kr, vr = c.host_pages()
        for dst, src in zip(parts(pages), parts(c.pages(host, gpu))):
            dst[:c.n_pages].copy_(src)
        for dst, src in ((seqs.table, c.table), (seqs.length, c.lens), (seqs.first, c.first)):
            dst.copy_(torch.from_numpy(src))
        q.copy_(c.q)
        g.replay()
        torch.cuda.synchronize()
        eager = cache.lsh_cache_attn_fwd(cfg, pages, seqs, q)
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])
        ref = C.attend(c.q.double().numpy(), kr, vr, host[4].astype(np.float64), c.first, c.lens, c.table, 16, 0.125, True, 1e5)
        compare(*eager, *ref, c)


# ---- whole prompts: the table no wider than their tokens ----


def check_sampled(c, gpu, tokens):
    """As check_attention, at some tokens alone: for the oracle each is the last of a sequence of its own that ends there."""
    host, kr, vr = c.host_pages()
    out, lse = cache.lsh_cache_attn_fwd(c.cfg, c.pages(host, gpu), c.seqs(gpu), c.q.to(gpu))
    torch.cuda.synchronize()
    s = np.searchsorted(c.first, tokens, side="right") - 1
    lens = (c.lens[s] - (c.first[s + 1] - tokens) + 1).astype(np.int32)
    ref = C.attend(c.q[tokens].double().numpy(), kr, vr, None if host[4] is None else host[4].astype(np.float64),
                   np.arange(len(tokens) + 1), lens, c.table[s], c.page, 0.125, c.shared, c.cfg.self_mask)
    compare(out[tokens], lse[tokens], *ref, c)


@pytest.mark.parametrize("type_", TYPES)
@pytest.mark.parametrize("heads", [(64, 64), (64, 8)])
def test_prompt_in_tiles_of_256(gpu, heads, type_):  # noqa: F811
    """One prompt of 2^17 rows: a workgroup for each tile of 256, keys not split."""
    H, Hkv = heads
    c = Case(type_, H == Hkv, H, Hkv, 64, [2100], [2100], seed=41)
    log("cache prompt", heads, type_)
    check_sampled(c, gpu, np.unique(np.concatenate([[0, 1, 62, 63, 64, 255, 256, 2098, 2099], c.rng.integers(0, c.T, 60)])))


@pytest.mark.parametrize("type_", TYPES)
@pytest.mark.parametrize("shared", [True, False])
def test_prompts_in_tiles_of_256_joined(gpu, shared, type_):  # noqa: F811
    """2^17 rows of prompts of unequal length: the long ones' keys are split and joined by sixteen lanes a row."""
    lens = [3000, 1, 17, 64, 700, 900, 1200, 1500, 1000, 64]
    c = Case(type_, shared, 16, 16 if shared else 4, 32, lens, lens, seed=42)
    assert c.T * c.H >= 1 << 17 and c.most * c.page < 2 * c.T
    log("cache prompts", shared, type_)
    edges = np.concatenate([c.first[:-1], c.first[1:] - 1])
    check_sampled(c, gpu, np.unique(np.concatenate([edges, c.rng.integers(0, c.T, 150)])))


@pytest.mark.parametrize("type_", TYPES)
@pytest.mark.parametrize("lens", [[1100], [300, 40, 1, 17, 299, 250, 64, 130]])
def test_prompts_in_tiles_of_64(gpu, lens, type_):  # noqa: F811
    """2^24 pairs and more, weights as one number: one prompt without parts, and several."""
    H = 16 if len(lens) == 1 else 64
    c = Case(type_, True, H, H, 16, lens, lens, seed=43)
    assert 1 << 24 <= c.T * H * c.most * 16 and c.T * H < 1 << 17
    log("cache prompts of 64 rows a tile", lens, type_)
    edges = np.concatenate([c.first[:-1], c.first[1:] - 1])
    check_sampled(c, gpu, np.unique(np.concatenate([edges, c.rng.integers(0, c.T, 40)])))


def large_prompt(c):
    """The case with a table of 2^24 pairs, less than twice as wide as its new tokens: tiles of 64 rows, one number a weight."""
    width = -(-(1 << 24) // (c.T * c.H * c.page))
    c.table = np.concatenate([c.table, np.full((len(c.lens), max(0, width - c.most)), c.n_pages, np.int32)], 1)
    c.most = max(c.most, width)
    c.cfg = replace(c.cfg, max_pages=c.most)
    assert c.most * c.page < 2 * c.T and c.T * c.H < 1 << 17
    return c


@pytest.mark.parametrize("shared", [True, False])
@pytest.mark.parametrize("type_", TYPES)
def test_prompts_in_tiles_of_64_hide_what_follows(gpu, type_, shared):  # noqa: F811
    """Holes, NaN in hidden rows, and infinities that some rows see; the rows that do not see them keep their bits."""
    def run(bad):
        c = Case(type_, shared, 64, 64 if shared else 32, 16, [100, 420], [60, 400], seed=44, fill="nan")
        c.table[1, 9] = -1
        for s, p in bad.items():
            at = c.table[s, p // 16], p % 16
            c.v[at[0], 1, at[1], 40] = np.inf
        host, _, _ = c.host_pages()
        large_prompt(c)
        return c, *cache.lsh_cache_attn_fwd(c.cfg, c.pages(host, gpu), c.seqs(gpu), c.q.to(gpu))

    bad = {0: 75, 1: 301}  # position of the bad row in each sequence
    log("cache prompts of 64 rows a tile, bad rows", type_, shared)
    (c, out, lse), (_, want, want_lse) = run(bad), run({})
    heads = slice(1, 2) if shared else slice(2, 4)
    assert torch.equal(lse, want_lse)
    for s, p in bad.items():
        n = p - (c.lens[s] - c.news[s]) + (1 if shared else 0)  # new tokens that do not see it
        wrong = want[c.first[s] + n:c.first[s + 1], heads]  # a block of codes with an infinity reads as NaN
        wrong[..., slice(40, 41) if type_ == "bf16" else slice(32, 64)] = np.inf if type_ == "bf16" else np.nan
    torch.testing.assert_close(out, want, rtol=0, atol=0, equal_nan=True)
    c = Case(type_, shared, 64, 64 if shared else 32, 16, [100, 420], [60, 400], seed=44, fill="nan")
    c.table[1, 9] = -1
    check_sampled(large_prompt(c), gpu, np.unique(np.concatenate([[0, 59, 60, 203, 204, 220, 459], c.rng.integers(0, 460, 40)])))


# ---- decoding ----


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("type_", TYPES)
def test_decoding_of_long_calls(gpu, type_, heads):  # noqa: F811
    """Tables for 2^24 pairs: 4-bit values take their weights as one number there."""
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 200, 1000, 5000, 0, 129]
    news = [1] * 11 + [0, 2]
    for shape in ("whole", "holes"):
        c = Case(type_, heads.startswith("shared"), *HEADS[heads], 16, lens, news, seed=51, fill="nan")
        if shape == "holes":
            c.table[8, 3], c.table[9, 0], c.table[10, 100:107], c.table[2, 0] = -1, c.n_pages, -9, -1
        log("cache decoding", type_, heads, shape)
        check_attention(widen(c, c.H // c.Hkv, 1 << 24), gpu)


@pytest.mark.parametrize("type_", TYPES)
@pytest.mark.parametrize("shared", [True, False])
def test_many_sequences_of_which_some_are_split(gpu, shared, type_):  # noqa: F811
    """More sequences than workgroups plan for themselves, some long enough to be split, chunks and single tokens."""
    rng = np.random.default_rng(61)
    lens = rng.integers(0, 60, 200)
    lens[rng.integers(0, 200, 12)] = rng.integers(1000, 3000, 12)
    news = np.minimum(rng.integers(0, 3, 200), lens)
    news[lens >= 1000] = rng.choice([1, 2, 20, 40, 90], (lens >= 1000).sum())
    log("cache many sequences split", shared, type_)
    check_attention(Case(type_, shared, 2, 2 if shared else 1, 16, lens, news, seed=62), gpu)
    c = Case(type_, shared, 2, 2 if shared else 1, 16, lens, news, seed=63)
    check_attention(tiles(c, 256), gpu)


@pytest.mark.parametrize("type_", TYPES)
def test_a_sequence_for_every_workgroup(gpu, type_):  # noqa: F811
    """2100 decoding sequences of 8 heads, a few of them long: parts of those alone, joined by sixteen lanes a row."""
    rng = np.random.default_rng(71)
    lens = rng.integers(1, 40, 2100)
    lens[rng.integers(0, 2100, 9)] = rng.integers(600, 2500, 9)
    log("cache sequence for every workgroup", type_)
    check_attention(Case(type_, True, 8, 8, 16, lens, np.ones(2100, int), seed=72, max_new=1), gpu)
