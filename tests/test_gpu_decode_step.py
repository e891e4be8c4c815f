"""A layer's decoding steps as a serving program runs them: the norm between blocks, 4-bit projections, rows into the
cache, attention over it, 4-bit products back onto the stream; prompts in chunks, then token by token, eager and captured.
Beside it the same layer from the calls that the library had: bf16 products of the unpacked matrices, norm and rotation,
cache write."""
import numpy as np
import pytest
import torch

from paper_2001_04451_amd import cache, lsh, qk, residual, w4

from gpu_common import log

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
H, DM, FF, PAGE = 4, 256, 512, 16  # heads with shared keys, widths, page


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    cache.lib()
    return torch.device("cuda:0")


class Layer:
    def __init__(self, gpu, kind, seed=0):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g).to(gpu)
        shapes = {"qv": (2 * H * 64, DM), "o": (DM, H * 64), "w1": (FF, DM), "w2": (DM, FF)}
        self.cfg = {n: w4.W4Config(N=a, K=b, type=kind[0], group=kind[1], zeros=kind[2]) for n, (a, b) in shapes.items()}
        self.packed = {n: w4.lsh_w4_quantize(self.cfg[n], r(a, b) / b ** 0.5) for n, (a, b) in shapes.items()}
        self.b1, self.b2 = 0.1 * r(FF), 0.1 * r(DM)
        self.gain, self.g1, self.g2, self.gp = (1 + 0.1 * r(n) for n in (64, DM, DM, DM))
        self.freq = torch.from_numpy((10000.0 ** (-np.arange(32) / 32)).astype(np.float32)).to(gpu)

    def step(self, x, ccfg, pages, seqs):
        """One step of T rows of the stream x [T, DM] fp32."""
        T = x.shape[0]
        N, Wt = residual.ResidualConfig, residual.ResidualWeights
        _, z = residual.lsh_residual_norm_fwd(N(T=T, D=DM, post=False), x, None, None, Wt(pre_g=self.g1))
        rows = w4.lsh_linear_w4(self.cfg["qv"], z, self.packed["qv"], dtype=BF)
        q = cache.lsh_cache_append(ccfg, qk.QkConfig(T=T, Hq=H), pages, seqs, rows, self.gain, None, self.freq)
        a, _ = cache.lsh_cache_attn_fwd(ccfg, pages, seqs, q)
        f = w4.lsh_linear_w4(self.cfg["o"], a.view(T, H * 64), self.packed["o"], dtype=BF)
        y, z2 = residual.lsh_residual_norm_fwd(N(T=T, D=DM), x, f, None, Wt(post_g=self.gp, pre_g=self.g2))
        h = w4.lsh_linear_w4(self.cfg["w1"], z2, self.packed["w1"], self.b1, relu=True, dtype=BF)
        out = w4.lsh_linear_w4(self.cfg["w2"], h, self.packed["w2"], self.b2, resid=y)
        return dict(z=z, rows=rows, q=q, a=a, f=f, y=y, z2=z2, h=h, out=out)

    def plain(self, s, x, ccfg, pages, seqs, pos):
        """Each stage again from the step's own inputs to it, in fp64 or by the library's earlier calls: {stage: (result,
        bound)}."""
        def rms(t, g):
            return t * torch.rsqrt(t.square().mean(-1, keepdim=True) + 1e-6) * g.double()

        def product(t, n):
            w = w4.lsh_w4_unpack(self.cfg[n], self.packed[n]).double()
            # the codes' own magnitudes, 8 + 7 steps to a scale, are what int4's sums reach on the way
            size = t.double().abs() @ (w.abs().amax(1, keepdim=True).expand_as(w) * 3).t()
            return t.double() @ w.t(), size * (w.shape[1] + 40) * 2.0 ** -24

        half = lambda ref, tol: (ref, tol + 2.0 ** -8 * ref.abs() * 1.01)
        f32 = 60 * 2.0 ** -24
        r = {}
        z = rms(x.double(), self.g1)
        r["z"] = half(z, f32 * z.abs())
        r["rows"] = half(*product(s["z"], "qv"))
        r["f"] = half(*product(s["a"].reshape(len(x), -1), "o"))
        y = x.double() + rms(s["f"].double(), self.gp)
        r["y"] = (y, f32 * (y.abs() + x.abs()))
        z2 = rms(s["y"].double(), self.g2)
        r["z2"] = half(z2, f32 * z2.abs())
        h, tol = product(s["z2"], "w1")
        r["h"] = half((h + self.b1).clamp(min=0), tol + 2.0 ** -23 * (h.abs() + 1))
        o, tol = product(s["h"], "w2")
        r["out"] = (s["y"].double() + (o + self.b2.double()), tol + 2.0 ** -22 * (o.abs() + s["y"].abs() + 1))
        # norm, rotation and write in the library's two calls, on the same rows in fp32: the same bits
        rows = s["rows"].float()
        q, _ = qk.lsh_qk_norm_rotate_fwd(qk.QkConfig(T=len(x), Hq=H), rows[:, :H * 64].contiguous(), self.gain, None,
                                         self.freq, pos)
        cache.lsh_cache_write(ccfg, pages, seqs, q, rows[:, H * 64:].reshape(-1, H, 64).contiguous())
        r["q"] = (q.to(BF).double(), torch.zeros_like(q, dtype=torch.float64))
        return r


KINDS = [("int4", 128, False), ("int4", 32, True), ("e2m1", 32, False)]


@pytest.mark.parametrize("type_", ["bf16", "e4m3", "e2m1"])
@pytest.mark.parametrize("kind", KINDS, ids=["int4", "int4-zeros", "e2m1"])
def test_layer(gpu, kind, type_):
    layer = Layer(gpu, kind)
    lens = [70, 33, 5]
    B, most = len(lens), 8
    table = torch.arange(B * most, dtype=torch.int32).flip(0).view(B, most).to(gpu)
    g = torch.Generator().manual_seed(7)
    x = [torch.randn(n + 4, DM, generator=g).to(gpu) for n in lens]
    pages = two = None
    at = [0] * B
    for step in ([40, 33, 5], [30, 0, 0], [1, 1, 1], [1, 1, 1], [0, 1, 1]):
        T = sum(step)
        log("layer", kind, type_, step)
        cfg = cache.CacheConfig(n_seq=B, T=T, H=H, Hkv=H, n_pages=B * most, max_pages=most, page=PAGE, type=type_,
                                max_new=max(step))
        if pages is None:
            pages, two = cache.Pages.empty(cfg, gpu), cache.Pages.empty(cfg, gpu)
            for a, b in ((pages.k, two.k), (pages.v, two.v), (pages.k_scale, two.k_scale), (pages.v_scale, two.v_scale),
                         (pages.k_inv, two.k_inv)):
                if a is not None:
                    a.zero_(), b.zero_()
        rows = torch.cat([t[a:a + n] for t, a, n in zip(x, at, step)])
        pos = torch.cat([torch.arange(a, a + n) for a, n in zip(at, step)]).to(torch.int32).to(gpu)
        at = [a + n for a, n in zip(at, step)]
        seqs = cache.Sequences(torch.tensor(np.concatenate([[0], np.cumsum(step)]), dtype=torch.int32, device=gpu),
                               torch.tensor(at, dtype=torch.int32, device=gpu), table)
        got = layer.step(rows, cfg, pages, seqs)
        ref = layer.plain(got, rows, cfg, two, seqs, pos)
        torch.cuda.synchronize()
        for n, (want, tol) in ref.items():
            err = (got[n].double() - want).abs()
            assert (err <= tol).all(), f"{n}: {(err / tol.clamp(min=1e-300)).max().item():.2f} of the bound"
        for n in ("k", "v", "k_scale", "v_scale", "k_inv"):
            a, b = getattr(pages, n), getattr(two, n)
            assert a is None or torch.equal(a, b), n


def test_layer_captured(gpu):
    """A decoding step captured once and replayed while the sequences grow; eager steps beside it on pages of their own."""
    layer = Layer(gpu, KINDS[0], seed=1)
    B, most, lens = 5, 4, [1, 9, 16, 17, 40]
    cfg = cache.CacheConfig(n_seq=B, T=B, H=H, Hkv=H, n_pages=B * most, max_pages=most, page=PAGE, type="e4m3", max_new=1)
    table = torch.arange(B * most, dtype=torch.int32).view(B, most).to(gpu)
    length = torch.tensor(lens, dtype=torch.int32, device=gpu)
    seqs = cache.Sequences(torch.arange(B + 1, dtype=torch.int32, device=gpu), length, table)
    pages, two = cache.Pages.empty(cfg, gpu), cache.Pages.empty(cfg, gpu)
    for p in (pages, two):
        for t in (p.k, p.v, p.k_scale, p.v_scale, p.k_inv):
            t.zero_()
    x = torch.randn(B, DM, device=gpu)
    log("layer captured")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        layer.step(x, cfg, pages, seqs)
    torch.cuda.current_stream().wait_stream(s)
    layer.step(x, cfg, two, seqs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = layer.step(x, cfg, pages, seqs)
    for _ in range(4):
        x.normal_()
        length.add_(1)
        graph.replay()
        want = layer.step(x, cfg, two, seqs)
        torch.cuda.synchronize()
        for n in got:
            assert torch.equal(got[n], want[n]), n
        assert torch.equal(pages.k, two.k) and torch.equal(pages.v, two.v)


def test_training_step(gpu):
    """The norm between blocks under the LSH attention's training step: forward through norm, attention and the sum, and
    back, against the same chain in fp64 around the attention's own gradients."""
    from paper_2001_04451_amd.lsh import Config
    Hh, L = 2, 256
    D, T = Hh * 64, L
    g = torch.Generator().manual_seed(3)
    x, f = torch.randn(T, D, generator=g).to(gpu), torch.randn(T, D, generator=g).bfloat16().to(gpu)
    wt = residual.ResidualWeights(post_g=(1 + 0.1 * torch.randn(D, generator=g)).to(gpu),
                                  pre_g=(1 + 0.1 * torch.randn(D, generator=g)).to(gpu))
    cfg = residual.ResidualConfig(T=T, D=D, eps=1e-6)
    y, z = residual.lsh_residual_norm_fwd(cfg, x, f, None, wt)
    q = z.view(L, Hh, 64).transpose(0, 1).contiguous().unsqueeze(0)
    acfg = Config(B=1, H=Hh, L=L, n_buckets=8, n_rounds=2, causal=True)
    R = torch.randn(2, 64, 4, generator=g).to(gpu)
    st = lsh.lsh_attention_fwd(acfg, q, q, R)
    dout = torch.randn(1, Hh, L, 64, generator=g).bfloat16().to(gpu)
    dq, dv = lsh.lsh_chunk_attn_bwd(acfg, q, q, st.out, dout, st.lse, st.buckets, st.perm, st.undo, st.bstart)
    dz = (dq + dv)[0].transpose(0, 1).reshape(T, D).contiguous()
    dy = torch.randn(T, D, generator=g).to(gpu)
    grads = residual.lsh_residual_norm_bwd(cfg, y, f, None, wt, dy, dz)
    torch.cuda.synchronize()
    X, F, P, Q = (t.double().cpu().requires_grad_() for t in (x, f, wt.post_g, wt.pre_g))
    rms = lambda t: t / (t.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt()
    Y = X + rms(F) * P
    ((Y * dy.double().cpu()).sum() + (rms(Y) * Q * dz.double().cpu()).sum()).backward()
    for n, t in (("dx", X), ("df", F), ("dpost_g", P), ("dpre_g", Q)):
        want = t.grad
        # fp32 through two norms, and a forward whose y was rounded: some tens of half steps of what is summed
        assert ((grads[n].double().cpu() - want).abs() <= 200 * 2.0 ** -24 * (want.abs() + want.abs().max())).all(), n
