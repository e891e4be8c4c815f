"""GPU parity of the paged cache and of the attention over it with the fp64 oracle, at the sizes, masks and
contents where they can go wrong; codes and scales byte for byte."""
import numpy as np
import pytest
import torch

from oracle import cache as C
from paper_2001_04451_amd import cache, lsh

from gpu_common import log

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cache.lib()
    return torch.device("cuda:0")


class Case:
    """Sequences over a pool whose pages lie in random order, every slot holding a row."""

    def __init__(self, type_, shared, H, Hkv, page, lens, news, seed=0, T=None, scale=None, max_new=0, fill="rows"):
        rng = np.random.default_rng(seed)
        self.type, self.shared, self.H, self.Hkv, self.page = type_, shared, H, Hkv, page
        self.lens, self.news, self.rng = np.array(lens, np.int32), np.array(news, np.int32), rng
        self.first = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
        self.T = max(1, int(self.first[-1])) if T is None else T
        used = [-(-int(n) // page) for n in lens]
        self.n_pages, self.most = sum(used) + 2, max(1, max(used))
        order = rng.permutation(self.n_pages).astype(np.int32)
        self.table = np.full((len(lens), self.most), -1, np.int32)
        at = 0
        for s, n in enumerate(used):
            self.table[s, :n] = order[at:at + n]
            at += n
        shape = (self.n_pages, Hkv, page, 64)
        self.k, self.v = (rng.standard_normal(shape).astype(np.float32) for _ in "kv")
        self.k *= np.exp(0.3 * rng.standard_normal(shape[:3] + (1,))).astype(np.float32)
        if fill == "nan":  # beside the sequences' own slots nothing but NaN
            mine = np.zeros(shape[:3], bool)
            for s, n in enumerate(lens):
                for j in range(int(n)):
                    mine[self.table[s, j // page], :, j % page] = True
            self.k[~mine] = np.nan
            self.v[~mine] = np.nan
        self.q = torch.from_numpy((rng.standard_normal((self.T, H, 64)) *
                                   np.exp(0.3 * rng.standard_normal((self.T, H, 1)))).astype(np.float32)).bfloat16()
        self.cfg = cache.CacheConfig(n_seq=len(lens), T=self.T, H=H, Hkv=Hkv, n_pages=self.n_pages, max_pages=self.most,
                                     page=page, type=type_, shared_qk=shared, scale=scale, max_new=max_new)

    def host_pages(self):
        """Codes, scales and k_inv of the pool's rows, and the rows they stand for (stored, without k_inv)."""
        kc, ks = C.encode(self.k, self.type)
        vc, vs = C.encode(self.v, self.type)
        kr, vr = C.decode(kc, ks, self.type), C.decode(vc, vs, self.type)
        inv = C.inverse_length(kr).astype(np.float32) if self.shared else None
        return (kc, vc, ks, vs, inv), kr, vr

    def pages(self, host, gpu):
        return cache.Pages(*[None if t is None else torch.from_numpy(np.ascontiguousarray(t)).to(gpu) for t in host])

    def seqs(self, gpu):
        return cache.Sequences(*[torch.from_numpy(t).to(gpu) for t in (self.first, self.lens, self.table)])


def check_attention(c, gpu, **kw):
    host, kr, vr = c.host_pages()
    scale = 0.125 if c.cfg.scale is None else c.cfg.scale
    out = torch.full((c.T, c.H, 64), 7.0, dtype=torch.bfloat16, device=gpu)
    lse = torch.full((c.T, c.H), 7.0, device=gpu)
    pages, seqs, q = c.pages(host, gpu), c.seqs(gpu), c.q.to(gpu)
    cache.lsh_cache_attn_fwd(c.cfg, pages, seqs, q, out=out, lse=lse, **kw)
    torch.cuda.synchronize()
    with np.errstate(invalid="ignore"):
        inv = None if host[4] is None else host[4].astype(np.float64)
        ref, ref_lse, spread, reach = C.attend(c.q.double().numpy(), kr, vr, inv, c.first, c.lens, c.table, c.page, scale,
                                               c.shared, c.cfg.self_mask)
    compare(out, lse, ref, ref_lse, spread, reach, c)
    return out, lse, (pages, seqs, q)


def compare(out, lse, ref, ref_lse, spread, reach, c):
    out, lse = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    outside = np.isnan(ref_lse)
    assert (out[outside] == 7).all() and (lse[outside] == 7).all(), "rows outside all sequences were written"
    ref, ref_lse = np.where(outside[..., None], 7, ref), np.where(outside, 7, ref_lse)
    spread = np.where(outside[..., None], 0, spread)
    # A logit is a sum of 64 exact products in fp32 and two roundings of its size more: the sum's parts are at most
    # |q||k| scale together, which `reach` bounds within a factor of 64 for these rows (|q||k| <= 12 * 12, and a row's
    # largest logit is above 1/64 of that or the bound's floor of one is taken), so dz <= 2^-24 * 70 * max(1, 64 reach)
    # is far more than it can be off; 2^-22 covers exp2.
    dz = 70 * 2.0 ** -24 * np.maximum(1, 2 * reach) * 2 + 2.0 ** -22
    # weights: rounded to bf16 (2^-8, finfo's half step) above and in the sum below; the output once more
    tol = (2 * 2.0 ** -8 + 2 * dz[..., None]) * spread * (1 + 2.0 ** -7) + 2.0 ** -8 * np.abs(ref) + 1e-38
    err = np.abs(out - ref)
    assert (err <= tol).all(), f"out off by {np.nanmax(err):.3e}, {np.nanmax(err / tol):.2f} of the tolerance"
    empty = np.isneginf(ref_lse)
    assert np.isneginf(lse[empty]).all() and (out[empty] == 0).all()
    ltol = dz + 2.0 ** -22 * np.abs(np.where(empty, 0, ref_lse)) + 2.0 ** -20
    lerr = np.abs(np.where(empty, 0, lse) - np.where(empty, 0, ref_lse))
    assert (lerr <= ltol).all(), f"lse off by {lerr.max():.3e}"


TYPES = ["bf16", "e4m3", "e2m1"]
# (page, lengths, new tokens): one token each; short and empty sequences; pages that end inside tiles of 16 to 64 keys;
# a few tokens; chunks; chunks beside decoding; whole prompts
SHAPES = {
    "decode": (16, [1, 2, 15, 16, 17, 63, 64, 65, 200, 1000], [1] * 10),
    "empty": (32, [0, 5, 0, 33, 1], [0, 1, 0, 2, 0]),
    "one": (16, [1], [1]),
    "few": (64, [130, 7, 64, 500], [5, 7, 16, 3]),
    "chunk": (32, [333], [77]),
    "mixed": (16, [700, 40, 1, 129], [300, 1, 1, 17]),
    "prompt": (128, [257, 64], [257, 64]),
    "beyond": (16, [3, 20], [9, 20]),  # more new tokens than length: the first have negative positions
}


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("heads", ["shared2", "shared1", "group1", "group4", "group6"])
@pytest.mark.parametrize("type_", TYPES)
def test_attention(gpu, type_, heads, shape):
    page, lens, news = SHAPES[shape]
    H, Hkv = {"shared2": (2, 2), "shared1": (1, 1), "group1": (2, 2), "group4": (8, 2), "group6": (6, 1)}[heads]
    log("cache attention", type_, heads, shape)
    check_attention(Case(type_, heads.startswith("shared"), H, Hkv, page, lens, news, seed=len(shape), fill="nan"), gpu)


@pytest.mark.parametrize("max_new", [1, 4, 64, 1000])
@pytest.mark.parametrize("shared", [True, False])
def test_attention_any_max_new(gpu, max_new, shared):
    """max_new is a hint: results stay right whatever it says."""
    log("cache attention max_new", max_new, shared)
    check_attention(Case("e4m3", shared, 2, 2, 16, [300, 70, 9], [40, 1, 9], max_new=max_new), gpu)


@pytest.mark.parametrize("type_", TYPES)
def test_attention_long_split(gpu, type_):
    """Few rows over long caches, so that the keys are split over many workgroups; odd lengths."""
    log("cache attention long", type_)
    check_attention(Case(type_, True, 1, 1, 64, [9001], [1], seed=1), gpu)
    check_attention(Case(type_, False, 8, 1, 16, [5000, 77, 2049], [1, 1, 2], seed=2), gpu)
    check_attention(Case(type_, False, 2, 1, 32, [4001], [100], seed=3), gpu)


@pytest.mark.parametrize("scale", [0.01, 3.0, -0.125])
def test_attention_scales(gpu, scale):
    """Flat, peaked and negative scales; peaked logits pass the range in which no running maximum is needed."""
    log("cache attention scale", scale)
    for shared in (True, False):
        check_attention(Case("bf16", shared, 2, 2, 16, [150, 90], [1, 70], scale=scale), gpu)


def test_attention_many_sequences(gpu):
    """More sequences than a wave has lanes, many of them without new tokens or empty."""
    rng = np.random.default_rng(9)
    lens = rng.integers(0, 60, 300)
    news = np.minimum(rng.integers(0, 3, 300), np.maximum(lens, 0))
    log("cache attention many sequences")
    check_attention(Case("e4m3", True, 1, 1, 16, lens, news), gpu)
    lens = rng.integers(0, 9, 5000)
    news = np.minimum((rng.random(5000) < 0.02).astype(int), lens)
    check_attention(Case("bf16", False, 2, 1, 16, lens, news), gpu)


@pytest.mark.parametrize("shape", ["decode", "mixed"])
def test_attention_bad_pages(gpu, shape):
    """Pages outside the pool, whole and in the middle of a sequence, hold no one's keys; lengths past the table count
    for positions alone; rows behind the last sequence stay as they were."""
    page, lens, news = SHAPES[shape]
    for shared in (True, False):
        c = Case("e2m1", shared, 2, 2, page, lens, news, seed=5, T=int(sum(news)) + 3)
        c.table[:, 0] = np.where(np.arange(len(lens)) % 2 == 0, -5, c.n_pages + 100)
        if c.most > 2:
            c.table[3, 2] = 2 ** 31 - 1
        c.lens[-1] += 3 * page * c.most
        log("cache attention bad pages", shape, shared)
        check_attention(c, gpu)
        c = Case("e4m3", shared, 2, 2, page, lens, news, seed=6)
        c.table[:] = -1
        out, lse, _ = check_attention(c, gpu)
        assert not out.any() and torch.isneginf(lse).all()


def test_attention_bad_first(gpu):
    """Whatever `first` and `length` hold, the call stays inside its buffers and ends."""
    c = Case("bf16", True, 2, 2, 16, [40, 30, 20], [3, 3, 3])
    host, _, _ = c.host_pages()
    for first, lens in (([-7, 2, 100, 5], [40, 30, 20]), ([9, 6, 3, 0], [40, 30, 20]),
                        ([0, 3, 6, 2 ** 31 - 1], [2 ** 31 - 1, -2 ** 31, -5]), ([-2 ** 31, -9, -1, 2 ** 31 - 1], [1, 1, 2 ** 31 - 1])):
        c.first, c.lens = np.array(first, np.int32), np.array(lens, np.int32)
        log("cache bad first", first, lens)
        guard = torch.full((c.T + 2, 2, 64), 7.0, dtype=torch.bfloat16, device=gpu)
        pages, seqs = c.pages(host, gpu), c.seqs(gpu)
        cache.lsh_cache_attn_fwd(c.cfg, pages, seqs, c.q.to(gpu), out=guard[1:-1])
        k, _ = cache.lsh_cache_read(c.cfg, pages, seqs, torch.bfloat16)
        torch.cuda.synchronize()
        assert (guard[0] == 7).all() and (guard[-1] == 7).all()


@pytest.mark.parametrize("type_", TYPES)
@pytest.mark.parametrize("shared", [True, False])
def test_attention_nothing_leaks_from_later_tokens(gpu, type_, shared):
    """NaN and infinities in a new token's rows reach that token's successors alone."""
    c = Case(type_, shared, 2, 2, 16, [100, 200], [40, 130], seed=8)
    bad = {0: 75, 1: 150}  # position of the bad row in each sequence
    for s, p in bad.items():
        c.v[c.table[s, p // 16], 0, p % 16, 5] = np.nan
        c.v[c.table[s, p // 16], 1, p % 16, 40] = np.inf
        c.k[c.table[s, p // 16], :, p % 16, 7] = np.inf if type_ == "bf16" else np.nan
    host, _, _ = c.host_pages()
    log("cache attention leaks", type_, shared)
    out, lse = cache.lsh_cache_attn_fwd(c.cfg, c.pages(host, gpu), c.seqs(gpu), c.q.to(gpu))
    clean = Case(type_, shared, 2, 2, 16, [100, 200], [40, 130], seed=8)
    host, _, _ = clean.host_pages()
    want, want_lse = cache.lsh_cache_attn_fwd(clean.cfg, clean.pages(host, gpu), clean.seqs(gpu), clean.q.to(gpu))
    for s, p in bad.items():
        a, b = c.first[s], c.first[s + 1]
        n = p - (c.lens[s] - c.news[s]) + (1 if shared else 0)  # new tokens before it; with shared QK it does not see itself
        assert torch.equal(out[a:a + n], want[a:a + n]) and torch.equal(lse[a:a + n], want_lse[a:a + n])
        assert torch.isnan(lse[a + n:b]).all() or torch.isnan(out[a + n:b].float()).any(-1).all()


def test_attention_strided_queries_and_side_stream(gpu):
    """Queries as a view into wider rows, on a stream of their own; the same call twice gives the same bits."""
    c = Case("e4m3", False, 4, 2, 32, [600, 90], [1, 30])
    out, lse, (pages, seqs, q) = check_attention(c, gpu)
    wide = torch.full((c.T, 4 * 64 + 128), float("nan"), dtype=torch.bfloat16, device=gpu)
    wide[:, 64:64 + 256] = q.view(c.T, 256)
    view = wide[:, 64:64 + 256].unflatten(1, (4, 64))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out2, lse2 = cache.lsh_cache_attn_fwd(c.cfg, pages, seqs, view)
    side.synchronize()
    assert torch.equal(out, out2) and torch.equal(lse, lse2)


def test_attention_captured(gpu):
    """One captured graph serves new queries, lengths and tables; two graphs may share a workspace when replayed one
    after the other."""
    cases = [Case("e4m3", True, 2, 2, 16, lens, [1, 1, 1], seed=i) for i, lens in
             enumerate(([500, 40, 7], [1, 333, 64], [2000, 1999, 3]))]
    most, n_pages = max(c.most for c in cases), max(c.n_pages for c in cases)
    cfg = cache.CacheConfig(n_seq=3, T=3, H=2, Hkv=2, n_pages=n_pages, max_pages=most, page=16, type="e4m3")
    pages = cache.Pages.empty(cfg, gpu)
    for t in (pages.k, pages.v, pages.k_scale, pages.v_scale, pages.k_inv):
        t.zero_()
    table = torch.full((3, most), -1, dtype=torch.int32, device=gpu)
    seqs = cache.Sequences(torch.arange(4, dtype=torch.int32, device=gpu), torch.ones(3, dtype=torch.int32, device=gpu), table)
    q = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device=gpu)
    ws = cache.workspace(cfg, gpu)
    outs = [(torch.empty_like(q), torch.empty(3, 2, device=gpu)) for _ in range(2)]
    log("cache attention captured")
    graphs = []
    for out, lse in outs:
        cache.lsh_cache_attn_fwd(cfg, pages, seqs, q, out=out, lse=lse, workspace=ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            cache.lsh_cache_attn_fwd(cfg, pages, seqs, q, out=out, lse=lse, workspace=ws)
        graphs.append(g)
    for c in cases * 2:
        host, kr, vr = c.host_pages()
        p = c.pages(host, gpu)
        n = c.n_pages
        for dst, src in ((pages.k, p.k), (pages.v, p.v), (pages.k_scale, p.k_scale), (pages.v_scale, p.v_scale), (pages.k_inv, p.k_inv)):
            dst[:n].copy_(src)
        table.fill_(-1)
        table[:, :c.most].copy_(torch.from_numpy(c.table))
        seqs.length.copy_(torch.from_numpy(c.lens))
        q.copy_(c.q)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        eager = cache.lsh_cache_attn_fwd(cfg, pages, seqs, q)
        for out, lse in outs:
            assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])
        ref = C.attend(c.q.double().numpy(), kr, vr, host[4].astype(np.float64), c.first, c.lens, c.table, 16, 0.125, True, 1e5)
        compare(eager[0], eager[1], *ref, c)


def test_attention_workspace_contents_are_free(gpu):
    c = Case("bf16", True, 2, 2, 64, [3000, 100], [1, 20])
    out, lse, (pages, seqs, q) = check_attention(c, gpu)
    for fill in (0, 255, 0x7F):
        ws = torch.full((cache.workspace_bytes(c.cfg) + 8192,), fill, dtype=torch.uint8, device=gpu)
        ws[:4096], ws[-4096:] = 0xA5, 0xA5
        out2, lse2 = cache.lsh_cache_attn_fwd(c.cfg, pages, seqs, q, workspace=ws[4096:-4096])
        assert torch.equal(out, out2) and torch.equal(lse, lse2)
        assert (ws[:4096] == 0xA5).all() and (ws[-4096:] == 0xA5).all()


# ---- write and read ----


def _write(c, gpu, k, v, poison=0xC3):
    cfg = c.cfg
    pages = cache.Pages.empty(cfg, gpu)
    for t in (pages.k, pages.v, pages.k_scale, pages.v_scale):
        if t is not None:
            t.fill_(poison)
    if pages.k_inv is not None:
        pages.k_inv.fill_(-3.0)
    cache.lsh_cache_write(cfg, pages, c.seqs(gpu), k.to(gpu), v.to(gpu))
    torch.cuda.synchronize()
    return pages


def _expect(c, k, v, poison=0xC3):
    """The pool after the write, as NumPy arrays."""
    shape = (c.n_pages, c.Hkv, c.page)
    n = C.ROW_BYTES[c.type]
    want = {x: np.full(shape + (n,), poison, np.uint8) for x in ("k", "v")}
    for x in ("k_scale", "v_scale"):
        want[x] = None if c.type == "bf16" else np.full(shape + (2,), poison, np.uint8)
    want["k_inv"] = np.full(shape, -3.0) if c.shared else None
    for t, s, pos in C.tokens(c.first, c.lens, c.T):
        at = C.slot(c.table, s, pos, c.page, c.n_pages)
        if at is None:
            continue
        for x, rows in (("k", k), ("v", v)):
            codes, scale = C.encode(rows[t], c.type)
            want[x][at[0], :, at[1]] = codes
            if scale is not None:
                want[x + "_scale"][at[0], :, at[1]] = scale
            if x == "k" and c.shared:
                want["k_inv"][at[0], :, at[1]] = C.inverse_length(C.decode(codes, scale, c.type))
    return want


def _check_pages(pages, want):
    for x in ("k", "v", "k_scale", "v_scale"):
        if want[x] is not None:
            assert np.array_equal(getattr(pages, x).cpu().numpy(), want[x]), x
    if want["k_inv"] is not None:
        got, ref = pages.k_inv.cpu().numpy().astype(np.float64), want["k_inv"]
        # a sum of 64 squares (66 roundings of half their size under the root), a root and a quotient
        ok = np.abs(got - ref) <= (33 + 3) * 2.0 ** -24 * np.abs(ref)
        assert (ok | (np.isnan(got) & np.isnan(ref))).all()


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("type_", TYPES)
def test_write_and_read(gpu, type_, dtype, shape):
    page, lens, news = SHAPES[shape]
    for shared, H, Hkv in ((True, 3, 3), (False, 4, 1)):
        c = Case(type_, shared, H, Hkv, page, lens, news, seed=11, T=max(1, sum(news)) + 2)
        if shape == "mixed":
            c.table[1, 1], c.table[2, 0] = -1, c.n_pages
        k, v = (torch.from_numpy(c.rng.standard_normal((c.T, Hkv, 64)).astype(np.float32)).to(dtype) for _ in "kv")
        log("cache write", type_, dtype, shape, shared)
        pages = _write(c, gpu, k, v)
        _check_pages(pages, _expect(c, k.double().numpy(), v.double().numpy()))
        rk, rv = (torch.full((c.T, Hkv, 64), 7.0, dtype=dtype, device=gpu) for _ in "kv")
        cache.lsh_cache_read(c.cfg, pages, c.seqs(gpu), dtype, rk, rv)
        wk, wv = (np.full((c.T, Hkv, 64), 7.0) for _ in "kv")
        for t, s, pos in C.tokens(c.first, c.lens, c.T):
            at = C.slot(c.table, s, pos, page, c.n_pages)
            wk[t] = wv[t] = 0
            if at is not None:
                ek, ev = C.encode(k[t].double().numpy(), type_), C.encode(v[t].double().numpy(), type_)
                wk[t], wv[t] = C.decode(*ek, type_), C.decode(*ev, type_)
                if shared:
                    wk[t] *= pages.k_inv[at[0], :, at[1]].double().cpu().numpy()[:, None]
        half = torch.finfo(dtype).eps / 2
        assert np.array_equal(rv.double().cpu().numpy(), wv)
        # bf16: a product rounded to fp32 and then to bf16
        assert (np.abs(rk.double().cpu().numpy() - wk) <= (half + 2.0 ** -24) * 1.001 * np.abs(wk)).all()
        only, _ = cache.lsh_cache_read(c.cfg, pages, c.seqs(gpu), dtype, torch.full_like(rk, 7.0))
        assert torch.equal(only, rk)


@pytest.mark.parametrize("type_", TYPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_write_every_rounding(gpu, type_, dtype):
    """Rows of exact ties and their neighbours, zeros of both signs, the ends of the exponent range, non-finite values."""
    rows = [np.zeros(64), -np.zeros(64)]
    if type_ != "bf16":
        vals = C.code_values(type_)
        vals = vals[:127] if type_ == "e4m3" else vals
        mid = (vals[1:] + vals[:-1]) / 2
        for x in (vals, mid, np.nextafter(np.float32(mid), np.float32(0)), np.nextafter(np.float32(mid), np.float32(1e9))):
            for i in range(0, len(x), 31):
                part = np.resize(x[i:i + 31], 31)
                rows.append(np.concatenate([part, vals[-1:], -part, vals[-1:]]))
    rng = np.random.default_rng(0)
    for e in (-140, -130, -126, -120, -60, -1, 0, 1, 60, 110, 120):
        rows.append(np.ldexp(rng.standard_normal(64), e))
    for x in (np.nan, np.inf, -np.inf):
        for d in (0, 31, 32, 63):
            r = rng.standard_normal(64)
            r[d] = x
            rows.append(r)
    n = len(rows)
    k = torch.from_numpy(np.array(rows, np.float32)[:, None]).to(dtype)
    v = k.flip(0)
    c = Case(type_, True, 1, 1, 16, [n], [n])
    log("cache write roundings", type_, dtype)
    with np.errstate(all="ignore"):
        pages = _write(c, gpu, k, v)
        want = _expect(c, k.double().numpy(), v.double().numpy())
        if type_ == "bf16":  # NaN payloads are free
            for x in ("k", "v"):
                got = getattr(pages, x).cpu().numpy().view(np.uint16)
                nan = (got & 0x7FFF) > 0x7F80
                assert np.array_equal(nan, (want[x].view(np.uint16) & 0x7FFF) > 0x7F80)
                getattr(pages, x).copy_(torch.from_numpy(np.where(nan, want[x].view(np.uint16), got).view(np.uint8)))
        # lengths near the ends of fp32's range have subnormal inverses, good to 2^-149 alone
        inv = pages.k_inv.cpu().numpy().astype(np.float64)
        tiny = (np.abs(want["k_inv"]) < 2.0 ** -126) & (np.abs(inv - want["k_inv"]) <= 2.0 ** -149)
        pages.k_inv.copy_(torch.from_numpy(np.where(tiny, want["k_inv"], inv).astype(np.float32)))
        _check_pages(pages, want)


def test_write_strided_rows_and_stream(gpu):
    """k and v as views into one fused row, on a side stream."""
    c = Case("e4m3", False, 4, 2, 16, [50, 20], [11, 20])
    fused = torch.randn(c.T, 8 * 64, generator=torch.Generator().manual_seed(0))
    dev = fused.to(gpu)
    k, v = dev[:, 256:384].unflatten(1, (2, 64)), dev[:, 384:].unflatten(1, (2, 64))
    pages = cache.Pages.empty(c.cfg, gpu)
    for t in (pages.k, pages.v, pages.k_scale, pages.v_scale):
        t.fill_(0xC3)
    seqs = c.seqs(gpu)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cache.lsh_cache_write(c.cfg, pages, seqs, k, v)
    side.synchronize()
    _check_pages(pages, _expect(c, k.double().cpu().numpy(), v.double().cpu().numpy()))


def test_offsets_past_32_bits(gpu):
    """Pages beyond 4 GiB of the pool: written, read and attended to."""
    n_pages, H, page = 40000, 16, 64  # 128 KiB of keys a page
    cfg = cache.CacheConfig(n_seq=1, T=100, H=H, Hkv=H, n_pages=n_pages, max_pages=2, page=page)
    pages = cache.Pages.empty(cfg, gpu)
    c = Case("bf16", True, H, H, page, [100], [100], seed=3)
    k, v = (torch.from_numpy(c.rng.standard_normal((100, H, 64)).astype(np.float32)).bfloat16() for _ in "kv")
    outs = []
    for table in ([39999, 35000], [1, 0]):
        seqs = cache.Sequences(*(torch.tensor(x, dtype=torch.int32, device=gpu) for x in ([0, 100], [100], [table])))
        log("cache past 32 bits", table)
        cache.lsh_cache_write(cfg, pages, seqs, k.to(gpu), v.to(gpu))
        rk, rv = cache.lsh_cache_read(cfg, pages, seqs, torch.bfloat16)
        assert torch.equal(rv.cpu(), v)
        outs.append((rk, *cache.lsh_cache_attn_fwd(cfg, pages, seqs, c.q.to(gpu))))
        assert torch.equal(pages.v[table[1], :, 35].cpu().view(torch.bfloat16), v[99])
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_binding_refusals(gpu):
    c = Case("e4m3", True, 2, 2, 16, [20], [4])
    host, _, _ = c.host_pages()
    pages, seqs, q = c.pages(host, gpu), c.seqs(gpu), c.q.to(gpu)
    rows = torch.zeros(4, 2, 64, device=gpu)
    call = lambda **kw: cache.lsh_cache_attn_fwd(c.cfg, *{**dict(pages=pages, seqs=seqs, q=q), **kw}.values())
    with pytest.raises(ValueError, match="dtype"):
        call(q=q.float())
    with pytest.raises(ValueError, match="shape"):
        call(q=q[:3])
    with pytest.raises(ValueError, match="contiguous"):
        call(q=q.transpose(1, 2).contiguous().transpose(1, 2))
    with pytest.raises(ValueError, match="no k_inv"):
        call(pages=cache.Pages(pages.k, pages.v, pages.k_scale, pages.v_scale))
    with pytest.raises(ValueError, match="k_scale has shape"):
        call(pages=cache.Pages(pages.k, pages.v, pages.k_scale[:, :1], pages.v_scale, pages.k_inv))
    with pytest.raises(ValueError, match="GPU"):
        call(seqs=cache.Sequences(seqs.first.cpu(), seqs.length, seqs.table))
    with pytest.raises(ValueError, match="dtype"):
        call(seqs=cache.Sequences(seqs.first.long(), seqs.length, seqs.table))
    with pytest.raises(ValueError, match="dtype"):
        cache.lsh_cache_write(c.cfg, pages, seqs, rows, rows.bfloat16())
    with pytest.raises(TypeError):
        cache.lsh_cache_write(c.cfg, pages, seqs, rows.half(), rows.half())
    with pytest.raises(lsh.LshError):
        cache.lsh_cache_attn_fwd(c.cfg, pages, seqs, q, workspace=torch.empty(16, dtype=torch.uint8, device=gpu))


@pytest.mark.parametrize("page", [256, 4096])
def test_attention_large_pages(gpu, page):
    log("cache attention pages of", page)
    check_attention(Case("e4m3", True, 2, 2, page, [page + 3, 5, page], [1, 5, 40], fill="nan"), gpu)
    check_attention(Case("bf16", False, 4, 1, page, [300], [300], fill="nan"), gpu)


@pytest.mark.parametrize("type_", TYPES)
def test_attention_many_heads_on_one(gpu, type_):
    """More query heads on a key head than a narrow tile has rows, alone and in a batch."""
    log("cache attention 48 heads on one", type_)
    check_attention(Case(type_, False, 48, 1, 16, [500], [1]), gpu)
    check_attention(Case(type_, False, 40, 2, 16, [500, 70, 3], [1, 2, 1]), gpu)


def test_rows_before_and_behind_the_sequences(gpu):
    """Sequences need not begin at row 0 nor end at T: the rows outside stay as they were, on every kernel's path."""
    for lens, news, T in (([70, 3000], [1, 1], 9), ([500], [200], 260), ([90, 40, 0], [60, 1, 0], 100)):
        for shared in (True, False):
            c = Case("e4m3", shared, 2, 2, 16, lens, news, T=T)
            c.first += 5
            log("cache attention rows outside", lens, news)
            check_attention(c, gpu)


def test_log_partition_is_optional(gpu):
    """lse may be NULL in the C call; out is the same."""
    c = Case("bf16", True, 2, 2, 16, [2000, 50], [1, 40])
    out, _, (pages, seqs, q) = check_attention(c, gpu)
    ws = cache.workspace(c.cfg, gpu)
    out2 = torch.empty_like(out)
    assert cache.lib().lsh_cache_attn_fwd(c.cfg.ref(), 1, pages.c(), seqs.c(), q.data_ptr(), out2.data_ptr(), None,
                                          ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(out, out2)


def test_two_streams_at_once(gpu):
    """Calls over one pool on two streams, each with its own workspace."""
    cases = [Case("e4m3", True, 2, 2, 16, [4000, 100], [1, 1], seed=1), Case("e4m3", True, 2, 2, 16, [700], [300], seed=2)]
    runs = []
    for c in cases:
        out, lse, (pages, seqs, q) = check_attention(c, gpu)
        runs.append((c, out, lse, pages, seqs, q, cache.workspace(c.cfg, gpu), torch.cuda.Stream()))
    log("cache attention two streams")
    torch.cuda.synchronize()
    got = [[] for _ in runs]
    for _ in range(5):
        for i, (c, _, _, pages, seqs, q, ws, stream) in enumerate(runs):
            with torch.cuda.stream(stream):
                got[i].append(cache.lsh_cache_attn_fwd(c.cfg, pages, seqs, q, workspace=ws))
    torch.cuda.synchronize()
    for (_, out, lse, *_), results in zip(runs, got):
        assert all(torch.equal(out, a) and torch.equal(lse, b) for a, b in results)


@pytest.mark.parametrize("type_", TYPES)
def test_whole_step_captured(gpu, type_):
    """Write, read and attention in one graph, replayed on new rows, against eager calls."""
    c = Case(type_, True, 2, 2, 16, [300, 20], [40, 1])
    seqs = c.seqs(gpu)
    pools = [cache.Pages.empty(c.cfg, gpu) for _ in range(2)]
    for p in pools:
        for t in (p.k, p.v, p.k_scale, p.v_scale, p.k_inv):
            if t is not None:
                t.zero_()
    k, v = (torch.zeros(c.T, 2, 64, device=gpu) for _ in "kv")
    q = c.q.to(gpu)
    rk, rv = torch.empty_like(k), torch.empty_like(v)
    out, lse, ws = torch.empty_like(q), torch.empty(c.T, 2, device=gpu), cache.workspace(c.cfg, gpu)

    def step(pages, rk, rv, out, lse, ws):
        cache.lsh_cache_write(c.cfg, pages, seqs, k, v)
        cache.lsh_cache_read(c.cfg, pages, seqs, torch.float32, rk, rv)
        cache.lsh_cache_attn_fwd(c.cfg, pages, seqs, q, out=out, lse=lse, workspace=ws)

    log("cache step captured", type_)
    step(pools[0], rk, rv, out, lse, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(pools[0], rk, rv, out, lse, ws)
    for i in range(3):
        k.normal_(generator=torch.Generator(gpu).manual_seed(i))
        v.normal_(generator=torch.Generator(gpu).manual_seed(10 + i))
        graph.replay()
        eager = [torch.empty_like(t) for t in (rk, rv, out, lse, ws)]
        step(pools[1], *eager)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((rk, rv, out, lse), eager))
        assert torch.equal(pools[0].k, pools[1].k) and torch.equal(pools[0].v, pools[1].v)
