"""A cached context read back as rows for the LSH attention over all of it (one MI355X)."""
from dataclasses import replace

import pytest
import torch

from paper_2001_04451_amd import cache, lsh
from paper_2001_04451_amd import workloads as W

from gpu_common import log
from test_gpu_cache import gpu  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("type_", ["bf16", "e4m3", "e2m1"])
def test_lsh_attention_over_a_context_read_back(gpu, type_):  # noqa: F811
    """Read as separate keys the pages of a shared-QK cache give the query rows as stored, from which the LSH attention is
    computed; read as what it is, the same rows times 1 / their length."""
    w = W.WORKLOADS["causal_bf16_L16384"].scaled(B=1, H=2, L=512, n_buckets=8, n_rounds=2, seed=9)
    lc, (B, H, L) = lsh.Config.of(w), (w.B, w.H, w.L)
    g = torch.Generator().manual_seed(0)
    q, v = (torch.randn(L, H, 64, generator=g).bfloat16().to(gpu) for _ in "qv")
    cfg = cache.CacheConfig(n_seq=1, T=L, H=H, Hkv=H, n_pages=40, max_pages=32, page=16, type=type_)
    pages = cache.Pages.empty(cfg, gpu)
    seqs = cache.Sequences(*(torch.tensor(t, dtype=torch.int32, device=gpu) for t in ([0, L], [L], [list(range(39, 7, -1))])))
    cache.lsh_cache_write(cfg, pages, seqs, q, v)
    rq, rv = cache.lsh_cache_read(replace(cfg, shared_qk=False), pages, seqs, torch.bfloat16)
    log("cache context read back", type_)
    # stored values have at most four significant bits but for bf16's own: exact in bf16
    f, _ = cache.lsh_cache_read(replace(cfg, shared_qk=False), pages, seqs, torch.float32)
    assert torch.equal(rq.float(), f)
    if type_ == "bf16":
        assert torch.equal(rq, q) and torch.equal(rv, v)
    rk, _ = cache.lsh_cache_read(cfg, pages, seqs, torch.float32)
    unit = f.double() / f.double().norm(dim=-1, keepdim=True)
    # k_inv: a sum of 64 squares (66 roundings of half their size under the root), a root and a quotient; one product more
    assert ((rk.double() - unit).abs() <= (33 + 4) * 2.0 ** -24 * unit.abs()).all()
    R = torch.from_numpy(W.make_inputs(w)["R"]).to(gpu)
    heads = lambda t: t.transpose(0, 1).contiguous()[None]
    got = lsh.lsh_attention_fwd(lc, heads(rq), heads(rv), R)
    if type_ == "bf16":
        want = lsh.lsh_attention_fwd(lc, heads(q), heads(v), R)
        assert torch.equal(got.out, want.out) and torch.equal(got.buckets, want.buckets)
    assert got.out.isfinite().all() and got.out.shape == (B, H, L, 64)
