"""The per-head norm, the cache and its attention run together, as a model runs them: prompts in chunks and then
token by token, beside the dense attention over whole sequences; and a training step of the LSH attention behind the
norm."""
import numpy as np
import pytest
import torch

import oracle
from oracle import cache as C
from oracle import qk as Q
from paper_2001_04451_amd import cache, lsh, qk
from paper_2001_04451_amd import workloads as W

from gpu_common import log

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cache.lib()
    return torch.device("cuda:0")


def serve(gpu, type_, H, lens, steps, page=16, seed=0):
    """Feed B sequences of projected rows through norm, cache and attention in the given steps (tokens of each sequence
    a step); (q, v, out, lse) by sequence, [L][H][64]."""
    g = torch.Generator().manual_seed(seed)
    B = len(lens)
    x = [torch.randn(L, H * 64, generator=g).bfloat16().to(gpu) for L in lens]
    v = [torch.randn(L, H, 64, generator=g).bfloat16().to(gpu) for L in lens]
    gain = (1 + 0.1 * torch.randn(64, generator=g)).to(gpu)
    freq = torch.from_numpy((10000.0 ** (-np.arange(32) / 32)).astype(np.float32)).to(gpu)
    most = max(-(-L // page) for L in lens)
    table = torch.arange(B * most, dtype=torch.int32).flip(0).view(B, most).to(gpu)
    pages, at = None, [0] * B
    qs, outs, lses = ([[] for _ in lens] for _ in range(3))
    for step in steps:
        n = [min(s, L - a) for s, L, a in zip(step, lens, at)]
        T = sum(n)
        if T == 0:
            continue
        cfg = cache.CacheConfig(n_seq=B, T=T, H=H, Hkv=H, n_pages=B * most, max_pages=most, page=page, type=type_,
                                max_new=max(n))
        pages = cache.Pages.empty(cfg, gpu) if pages is None else pages
        new = [slice(a, a + k) for a, k in zip(at, n)]
        at = [a + k for a, k in zip(at, n)]
        first = torch.tensor(np.concatenate([[0], np.cumsum(n)]), dtype=torch.int32, device=gpu)
        seqs = cache.Sequences(first, torch.tensor(at, dtype=torch.int32, device=gpu), table)
        pos = torch.cat([torch.arange(s.start, s.stop) for s in new]).to(torch.int32).to(gpu)
        q, _ = qk.lsh_qk_norm_rotate_fwd(qk.QkConfig(T=T, Hq=H), torch.cat([a[s] for a, s in zip(x, new)]), gain, None,
                                         freq, pos)
        cache.lsh_cache_write(cfg, pages, seqs, q, torch.cat([a[s] for a, s in zip(v, new)]))
        out, lse = cache.lsh_cache_attn_fwd(cfg, pages, seqs, q)
        for lst, t in ((qs, q), (outs, out), (lses, lse)):
            for i, part in enumerate(t.split(n)):
                lst[i].append(part)
    torch.cuda.synchronize()
    return [[torch.cat(p) for p in lst] for lst in (qs, outs, lses)] + [v, x, gain, freq]


def test_chunks_then_tokens_is_dense_attention(gpu):
    """A bf16 cache fed in chunks of any size and then token by token: lsh_dense_attn_fwd over the whole sequences, and
    the oracle's, within the dense attention's tolerance."""
    lens = [301, 64, 17]
    steps = [[100, 40, 17], [1, 3, 0], [150, 20, 0], [7, 1, 0]] + [[1, 1, 0]] * 45
    log("serving against dense")
    qs, outs, lses, v, x, gain, freq = serve(gpu, "bf16", 4, lens, steps)
    for i, L in enumerate(lens):
        heads = lambda t: t.transpose(0, 1).contiguous()[None]  # [1][H][L][64]
        cfg = lsh.Config(B=1, H=4, L=L, n_buckets=2, n_rounds=1, causal=True)
        dense, dense_lse = lsh.lsh_dense_attn_fwd(cfg, heads(qs[i]), heads(v[i]))
        ref, ref_lse = oracle.dense_attn_fwd(heads(qs[i]).double().cpu().numpy(), heads(v[i]).double().cpu().numpy(), True)
        out, lse = heads(outs[i]), lses[i].t()[None]
        assert (out.float() - dense.float()).abs().max() <= 2e-2
        assert np.abs(out.double().cpu().numpy() - ref).max() <= 2e-2
        assert np.abs(lse.double().cpu().numpy() - ref_lse).max() <= 2e-2
        # and the rows are what the norm makes of the projections
        want = Q.norm_rotate(x[i].double().cpu().numpy().reshape(L, 4, 64), gain.double().cpu().numpy(), np.arange(L),
                             freq.double().cpu().numpy(), 64, False, 1e-6)
        got = qs[i].double().cpu().numpy()
        assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 1e-5 * np.abs(want).max(-1, keepdims=True)).all()


@pytest.mark.parametrize("type_", ["e4m3", "e2m1"])
def test_quantised_serving_is_attention_over_the_stored_rows(gpu, type_):
    """However the tokens were fed, each sees the rows that the cache stands for."""
    lens = [130, 33]
    log("serving quantised", type_)
    for steps in ([[130, 33]], [[64, 33], [1, 0], [65, 0]], [[1, 1]] * 130):
        qs, outs, lses, v, *_ = serve(gpu, type_, 2, lens, steps, page=32)
        for i, L in enumerate(lens):
            k, vv = qs[i].double().cpu().numpy(), v[i].double().cpu().numpy()
            k, vv = C.decode(*C.encode(k, type_), type_), C.decode(*C.encode(vv, type_), type_)
            pool = lambda r: r.transpose(1, 0, 2)[None]  # one page a sequence for the oracle
            inv = C.inverse_length(pool(k)).astype(np.float32).astype(np.float64)
            ref, ref_lse, spread, _ = C.attend(qs[i].double().cpu().numpy(), pool(k), pool(vv), inv, [0, L], [L],
                                               np.zeros((1, 1), np.int32), L, 0.125, True, 1e5)
            # two weight roundings and the output's, as in the attention's own tests, and 1e-4 for the logits
            tol = (2 * 2.0 ** -8 + 1e-4) * 1.01 * spread + 2.0 ** -8 * np.abs(ref)
            assert (np.abs(outs[i].double().cpu().numpy() - ref) <= tol).all()
            assert (np.abs(lses[i].double().cpu().numpy() - ref_lse) <= 1e-4 + 2e-7 * np.abs(ref_lse)).all()


def test_context_read_back_for_an_lsh_pass(gpu):
    """Cached keys read back are what the LSH attention hashes alike: buckets do not depend on a row's length."""
    lens, H = [512], 2
    log("serving read back")
    qs, *_ = serve(gpu, "bf16", H, lens, [[512]])
    cfg = cache.CacheConfig(n_seq=1, T=512, H=H, Hkv=H, n_pages=32, max_pages=32, page=16)
    pages = cache.Pages.empty(cfg, gpu)
    seqs = cache.Sequences(*(torch.tensor(t, dtype=torch.int32, device=gpu)
                             for t in ([0, 512], [512], [list(range(32))])))
    cache.lsh_cache_write(cfg, pages, seqs, qs[0], qs[0])
    k, v = cache.lsh_cache_read(cfg, pages, seqs, torch.float32)
    assert torch.equal(v, qs[0].float())
    assert ((k * k).sum(-1) - 1).abs().max() < 1e-5
    w = W.WORKLOADS["tiny_f32_L1024"].scaled(H=H, L=512, n_rounds=2)
    lc = lsh.Config.of(w)
    R = torch.from_numpy(W.make_inputs(w)["R"]).to(gpu)
    heads = lambda t: t.transpose(0, 1).contiguous()[None]
    a, b = lsh.lsh_hash(lc, heads(k), R), lsh.lsh_hash(lc, heads(v), R)
    # rounding the unit rows moves a projection by 2^-24 of the row: at most one row in thousands changes its bucket
    assert (a != b).sum() <= 2


def test_training_step_behind_the_norm(gpu):
    """x -> norm and rotation -> LSH attention -> its backward -> the norm's backward, against the formula on the very
    gradient that the attention gave; captured into a graph, twice, beside the eager step."""
    B, H, L = 2, 2, 256
    w = W.WORKLOADS["causal_bf16_L16384"].scaled(B=B, H=H, L=L, n_buckets=8, n_rounds=2, seed=7)
    cfg = lsh.Config.of(w)
    g = torch.Generator().manual_seed(1)
    x = torch.randn(B * L, H * 64, generator=g).bfloat16().to(gpu)
    v = torch.randn(B, H, L, 64, generator=g).bfloat16().to(gpu)
    dout = torch.randn(B, H, L, 64, generator=g).bfloat16().to(gpu)
    gain = (1 + 0.1 * torch.randn(64, generator=g)).to(gpu)
    freq = torch.from_numpy((10000.0 ** (-np.arange(32) / 32)).astype(np.float32)).to(gpu)
    R = torch.from_numpy(W.make_inputs(w)["R"]).to(gpu)
    qc = qk.QkConfig(T=B * L, Hq=H, L=L)

    def step():
        q, _ = qk.lsh_qk_norm_rotate_fwd(qc, x, gain, None, freq)
        st = lsh.lsh_attention_fwd(cfg, q, v, R)
        dq, dv = lsh.lsh_chunk_attn_bwd(cfg, q, v, st.out, dout, st.lse, st.buckets, st.perm, st.undo, st.bstart)
        dx, dgain, _ = qk.lsh_qk_norm_rotate_bwd(qc, x, gain, None, freq, None, dq)
        return st.out, dq, dv, dx, dgain

    log("training step")
    out, dq, dv, dx, dgain = eager = step()
    torch.cuda.synchronize()
    args = (x.double().cpu().numpy().reshape(B * L, H, 64), gain.double().cpu().numpy(), np.arange(B * L) % L,
            freq.double().cpu().numpy(), 64, False, 1e-6)
    d = Q.tokens_first(dq.double().cpu().numpy())
    ref, ref_gain, gain_abs = Q.norm_rotate_bwd(*args, d)
    n = np.abs(Q.norm_rotate(*args))
    size = np.abs(ref) + np.abs(d).max(-1, keepdims=True) * 4  # a value's terms: its gradient's pair and the mean's
    assert (np.abs(dx.double().cpu().numpy().reshape(B * L, H, 64) - ref) <= 200 * 2.0 ** -24 * size * (1 + n)).all()
    assert (np.abs(dgain.double().cpu().numpy() - ref_gain) <= 300 * 2.0 ** -24 * gain_abs).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        again = step()
        for a, b, c in zip(eager, captured, again):
            assert torch.equal(a, b) and torch.equal(a, c)
