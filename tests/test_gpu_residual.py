"""GPU parity of the step between two blocks, forward and backward, with the fp64 oracle, within the bounds of fp32
arithmetic that the oracle derives beside its results."""
import numpy as np
import pytest
import torch

from oracle import residual as R
from paper_2001_04451_amd import lsh, residual

from gpu_common import log

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    residual.lib()
    return torch.device("cuda:0")


class Case:
    def __init__(self, T, D, dtype=BF, norm="rms", post=True, pre=True, gate="none", scale=True, bias=True, alpha=1.0,
                 eps=1e-6, seed=0, offset=0.0, wide=0):
        rng = np.random.default_rng(seed)
        self.dtype, self.wide = dtype, wide
        self.cfg = residual.ResidualConfig(T=T, D=D, norm=norm, post=post, pre=pre, gate=gate, alpha=alpha, eps=eps)
        self.c = dict(layer=norm == "layer", gate=gate, post=post, pre=pre, eps=float(np.float32(eps)),
                      alpha=float(np.float32(alpha)))
        a = lambda *s: rng.standard_normal(s).astype(np.float32)
        self.x = a(T, D) * np.exp(a(T, 1)) + np.float32(offset)
        self.f = torch.from_numpy(a(T, D) * np.exp(a(T, 1)) + np.float32(offset)).to(dtype)
        self.gate = torch.from_numpy(3 * a(T, D)).to(dtype) if gate != "none" else None
        self.w = {"scale": 1 + np.float32(0.3) * a(D) if scale else None}
        for n, on in (("post", post), ("pre", pre)):
            self.w[n + "_g"] = 1 + np.float32(0.3) * a(D) if on else None
            self.w[n + "_b"] = a(D) if on and bias else None
        self.dy, self.dz = a(T, D), a(T, D) if pre else None

    def up(self, t, gpu, wide=0):
        """t on the GPU; with `wide`, as part of wider rows of NaN."""
        if t is None:
            return None
        t = (torch.from_numpy(t) if isinstance(t, np.ndarray) else t).to(gpu)
        if wide:
            rows = torch.full((t.shape[0], t.shape[1] + wide), float("nan"), dtype=t.dtype, device=gpu)
            rows[:, :t.shape[1]] = t
            return rows[:, :t.shape[1]]
        return t

    def weights(self, gpu):
        return residual.ResidualWeights(**{n: self.up(v, gpu) for n, v in self.w.items()})

    def wide64(self):
        d = lambda t: None if t is None else (t.astype(np.float64) if isinstance(t, np.ndarray) else t.double().numpy())
        return d(self.x), d(self.f), d(self.gate), {n: d(v) for n, v in self.w.items()}, d(self.dy), d(self.dz)


def close(name, got, ref, tol):
    got = got.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(ref)), name
    err = np.abs(got - ref)
    worst = np.nanmax(err / np.maximum(tol, 1e-300)) if err.size else 0
    assert (np.nan_to_num(err) <= np.nan_to_num(tol) + 1e-37).all(), f"{name} off by {np.nanmax(err):.3e}, {worst:.2f} of the bound"


def check(c, gpu):
    x, f, gate, w, dy, dz = c.wide64()
    F, G, weights = c.up(c.f, gpu, c.wide), c.up(c.gate, gpu, 3 * c.wide), c.weights(gpu)
    y, z = residual.lsh_residual_norm_fwd(c.cfg, c.up(c.x, gpu), F, G, weights)
    torch.cuda.synchronize()
    ref, tol = R.forward(c.c, x, f, gate, w)
    close("y", y, ref["y"], tol["y"])
    assert (z is None) == (not c.cfg.pre)
    if z is not None:
        half = torch.finfo(c.dtype).eps / 2 if c.dtype == BF else 0.0
        close("z", z, ref["z"], tol["z"] * (1 + half) + half * np.abs(ref["z"]))
    # the backward, at a y that both sides take as it is
    y32 = ref["y"].astype(np.float32)
    grads = residual.lsh_residual_norm_bwd(c.cfg, c.up(y32, gpu), F, G, weights, c.up(c.dy, gpu), c.up(c.dz, gpu))
    torch.cuda.synchronize()
    gref, gtol = R.backward(c.c, y32.astype(np.float64), f, gate, w, dy, dz)
    assert {n for n, t in grads.items() if t is not None} == set(gref)
    for n in gref:
        close(n, grads[n], gref[n], gtol[n])
    return y, z, grads


WIDTHS = [(1, 8), (3, 64), (5, 504), (9, 512), (7, 520), (300, 1000), (33, 1024), (6, 1032), (17, 2048), (5, 2056),
          (4, 4096), (2, 4104), (3, 8192)]


@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("T,D", WIDTHS)
def test_widths(gpu, T, D, norm):
    """A row of one thread, of a wave and one over, of two, four, eight and sixteen waves."""
    log("residual width", T, D, norm)
    check(Case(T, D, F32 if T % 2 else BF, norm, gate="sigmoid", seed=D), gpu)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("gate", ["none", "linear", "sigmoid"])
@pytest.mark.parametrize("post,pre", [(True, True), (True, False), (False, True), (False, False)])
@pytest.mark.parametrize("norm,bias,scale", [("rms", False, False), ("layer", True, True), ("rms", True, True),
                                             ("layer", False, False)])
def test_parts(gpu, norm, bias, scale, post, pre, gate, dtype):
    log("residual parts", norm, bias, scale, post, pre, gate, dtype)
    check(Case(37, 136, dtype, norm, post, pre, gate, scale, bias, alpha=-0.75, seed=3), gpu)


@pytest.mark.parametrize("T", [1, 2, 1023, 2049, 9000])
def test_many_rows(gpu, T):
    """More rows than workgroups hold at once; sums over all of them."""
    log("residual rows", T)
    check(Case(T, 72, BF, "layer", gate="sigmoid", seed=T), gpu)


@pytest.mark.parametrize("plain", [False, True])
@pytest.mark.parametrize("norm,post", [("rms", True), ("layer", True), ("rms", False)])
@pytest.mark.parametrize("T,D", [(9000, 264), (4500, 520), (2500, 1032), (1100, 2056), (600, 4104)])
def test_many_wide_rows(gpu, T, D, norm, post, plain):
    """Workgroups that walk over several rows, of one wave to sixteen: an even and an odd number of sums a row, with all
    weights and (`plain`) with gains alone; the same bits again."""
    log("residual wide rows", T, D, norm, post, plain)
    c = Case(T, D, F32 if plain else BF, norm, post, True, "sigmoid", scale=not plain, bias=not plain, seed=D)
    y, z, grads = check(c, gpu)
    F, G, w = c.up(c.f, gpu), c.up(c.gate, gpu), c.weights(gpu)
    y1, z1 = residual.lsh_residual_norm_fwd(c.cfg, c.up(c.x, gpu), F, G, w)
    assert torch.equal(y, y1) and torch.equal(z, z1)
    x, f, gate, w64, _, _ = c.wide64()
    y32 = R.forward(c.c, x, f, gate, w64)[0]["y"].astype(np.float32)
    again = residual.lsh_residual_norm_bwd(c.cfg, c.up(y32, gpu), F, G, w, c.up(c.dy, gpu), c.up(c.dz, gpu))
    for n, t in grads.items():
        assert (t is None and again[n] is None) or torch.equal(t, again[n]), n


@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_offset_rows(gpu, norm):
    """Rows whose mean is far from zero: the deviation is taken from the mean, not from squares."""
    log("residual offset", norm)
    check(Case(40, 520, F32, norm, gate="linear", seed=8, offset=1000.0), gpu)


@pytest.mark.parametrize("D", [64, 1032])
def test_strides(gpu, D):
    """f and gate as parts of wider rows, NaN beside them."""
    log("residual strides", D)
    check(Case(21, D, BF, "rms", gate="sigmoid", seed=5, wide=24), gpu)


def test_scales_of_rows(gpu):
    """Rows of 2^-50 and of 2^50, and zero rows with and without eps."""
    for power in (-50, 50):
        c = Case(6, 136, F32, "layer", gate="none", eps=0.0, seed=6)
        c.f = c.f * 2.0 ** power
        log("residual scale", power)
        check(c, gpu)
    for norm in ("rms", "layer"):
        c = Case(4, 136, F32, norm, gate="none", eps=0.0, bias=False, seed=7)
        c.f[1], c.x[1] = 0, 0
        y, z, grads = check(c, gpu)
        assert not z[1].any() and torch.equal(grads["dx"][1], c.up(c.dy, gpu)[1]) and not grads["df"][1].any()


def test_gate_ends(gpu):
    """Gates far out: 0 and 1 without NaN, and slopes that vanish."""
    c = Case(3, 64, F32, gate="sigmoid", seed=9)
    c.gate[0, :8] = torch.tensor([200.0, -200.0, 88.0, -88.0, 1e30, -1e30, float("inf"), -float("inf")])
    log("residual gates")
    y, _, grads = check(c, gpu)
    assert torch.isfinite(y).all() and torch.isfinite(grads["dgate"]).all()


def test_a_bad_row_stays_a_row(gpu):
    """NaN and infinities spoil their own row and the sums over rows, no other row."""
    c = Case(50, 520, BF, "layer", gate="sigmoid", seed=10)
    good = check(c, gpu)
    c.f[7, 3], c.gate[19, 500], c.x[33, 0] = float("nan"), float("inf"), np.inf
    F, G, w = c.up(c.f, gpu), c.up(c.gate, gpu), c.weights(gpu)
    y, z = residual.lsh_residual_norm_fwd(c.cfg, c.up(c.x, gpu), F, G, w)
    keep = [t for t in range(50) if t not in (7, 19, 33)]
    assert torch.equal(y[keep], good[0][keep]) and torch.equal(z[keep], good[1][keep])
    assert torch.isnan(z[7]).all() and torch.isnan(z[33]).all()


def test_without_a_branch(gpu):
    """The norm before the first block: y = x, z = pre(x); its backward."""
    c = Case(11, 1000, F32, "layer", post=False, gate="none", scale=False, seed=11)
    w, x = c.weights(gpu), c.up(c.x, gpu)
    log("residual without a branch")
    x64, _, _, w64, dy, dz = c.wide64()
    ref, tol = R.forward(c.c, x64, None, None, w64)
    for dtype in (F32, BF):
        y, z = residual.lsh_residual_norm_fwd(c.cfg, x, None, None, w, dtype=dtype)
        assert torch.equal(y, x) and z.dtype == dtype
        half = torch.finfo(dtype).eps / 2 if dtype == BF else 0.0
        close("z", z, ref["z"], tol["z"] * (1 + half) + half * np.abs(ref["z"]))
    for up_y in (c.dy, None):
        grads = residual.lsh_residual_norm_bwd(c.cfg, x, None, None, w, c.up(up_y, gpu), c.up(c.dz, gpu))
        gref, gtol = R.backward(c.c, x64, None, None, w64, None if up_y is None else dy, dz)
        assert {n for n, t in grads.items() if t is not None} == set(gref)
        for n in gref:
            close(n, grads[n], gref[n], gtol[n])


def test_without_a_stream(gpu):
    """x = NULL stands for zeros, dy = NULL for no gradient of y."""
    c = Case(11, 72, BF, gate="linear", seed=12)
    c.x[:] = 0
    F, G, w = c.up(c.f, gpu), c.up(c.gate, gpu), c.weights(gpu)
    y0, z0 = residual.lsh_residual_norm_fwd(c.cfg, c.up(c.x, gpu), F, G, w)
    y, z = residual.lsh_residual_norm_fwd(c.cfg, None, F, G, w)
    assert torch.equal(y, y0) and torch.equal(z, z0)
    zero = torch.zeros_like(y)
    a = residual.lsh_residual_norm_bwd(c.cfg, y, F, G, w, None, c.up(c.dz, gpu))
    b = residual.lsh_residual_norm_bwd(c.cfg, y, F, G, w, zero, c.up(c.dz, gpu))
    for n in a:
        assert (a[n] is None and b[n] is None) or torch.equal(a[n], b[n]), n


def test_alpha_takes_a_branch_off(gpu):
    """The reversible block's inverse: alpha = -1 gives x back, up to y's rounding."""
    c = Case(30, 264, F32, "layer", pre=False, gate="sigmoid", seed=13)
    F, G, w, x = c.up(c.f, gpu), c.up(c.gate, gpu), c.weights(gpu), c.up(c.x, gpu)
    y, _ = residual.lsh_residual_norm_fwd(c.cfg, x, F, G, w)
    back, _ = residual.lsh_residual_norm_fwd(
        residual.ResidualConfig(T=30, D=264, norm="layer", pre=False, gate="sigmoid", alpha=-1.0), y, F, G, w)
    # both sums round once, of the same branch
    assert ((back - x).abs() <= 2.0 ** -24 * (y.abs() + back.abs()) * 1.01).all()


def test_streams_graphs_and_guards(gpu):
    """Another stream, captured and replayed with eager calls between, workspaces of any content, canaries beside every
    output; repeated calls give the same bits."""
    c = Case(700, 200, BF, "layer", gate="sigmoid", seed=14)
    F, G, w, x = c.up(c.f, gpu), c.up(c.gate, gpu), c.weights(gpu), c.up(c.x, gpu)
    dy, dz = c.up(c.dy, gpu), c.up(c.dz, gpu)
    y0, z0 = residual.lsh_residual_norm_fwd(c.cfg, x, F, G, w)
    g0 = residual.lsh_residual_norm_bwd(c.cfg, y0, F, G, w, dy, dz)

    def guarded(like):
        buf = torch.full((like.numel() + 128,), 7.0, dtype=like.dtype, device=gpu)
        return buf, buf[64:-64].view(like.shape)

    y, z = guarded(y0), guarded(z0)
    outs = {n: guarded(t) for n, t in g0.items()}
    ws = torch.full((residual.workspace_bytes(c.cfg) + 512,), 255, dtype=torch.uint8, device=gpu)
    part = ws[256:-256]

    def step():
        residual.lsh_residual_norm_fwd(c.cfg, x, F, G, w, y=y[1], z=z[1])
        residual.lsh_residual_norm_bwd(c.cfg, y[1], F, G, w, dy, dz, grads={n: t[1] for n, t in outs.items()}, workspace=part)

    def right():
        torch.cuda.synchronize()
        assert torch.equal(y[1], y0) and torch.equal(z[1], z0)
        for n, (buf, t) in outs.items():
            assert torch.equal(t, g0[n]), n
            assert (buf[:64] == 7).all() and (buf[-64:] == 7).all(), n
        assert (ws[:256] == 255).all() and (ws[-256:] == 255).all()

    log("residual streams")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        step()
    right()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        for buf, t in (y, z, *outs.values()):
            t.fill_(float("nan"))
        part.fill_(k)
        graph.replay()
        residual.lsh_residual_norm_bwd(c.cfg, y0, F, G, w, dy, dz)
        right()


def test_as_the_blocks_layer_norm(gpu):
    """Beside the reversible block: the norm that lsh_rev_feed_forward applies inside, by a product with the identity."""
    D, T = 128, 70
    g = torch.Generator().manual_seed(1)
    x = torch.randn(T, D, generator=g).to(gpu)
    gain, bias = (1 + 0.1 * torch.randn(D, generator=g)).to(gpu), torch.randn(D, generator=g).to(gpu)
    cfg = lsh.BlockConfig(attn=lsh.Config(B=1, H=2, L=T, n_buckets=2, n_rounds=1), d_ff=128, ln_eps=1e-5)
    eye = torch.eye(D, device=gpu).bfloat16()
    w = lsh.BlockWeights(ln2_g=gain, ln2_b=bias, w1=eye, b1=torch.zeros(D, device=gpu), w2=eye,
                         b2=torch.zeros(D, device=gpu), ln1_g=gain, ln1_b=bias, w_qk=eye, w_v=eye, w_o=eye,
                         R=torch.zeros(1, 64, 1, device=gpu))
    out = lsh.rev_feed_forward(cfg, w, x.view(1, T, D)).view(T, D)
    own = residual.ResidualConfig(T=T, D=D, norm="layer", post=False, eps=1e-5)
    _, z = residual.lsh_residual_norm_fwd(own, x, None, None, residual.ResidualWeights(pre_g=gain, pre_b=bias))
    # both round the same number to bf16, within fp32's error of each other: a step apart at most
    assert ((out - z.float().clamp(min=0)).abs() <= 2.0 ** -7 * z.float().abs() + 1e-6).all()


def test_exchanged_weights_refused(gpu):
    """A weight whose storage becomes bf16 after a first call (as a module's conversion does) is not read as fp32."""
    cfg = residual.ResidualConfig(T=3, D=64, pre=False)
    x, f = torch.ones(3, 64, device=gpu), torch.ones(3, 64, device=gpu, dtype=BF)
    weights = residual.ResidualWeights(post_g=torch.nn.Parameter(torch.ones(64, device=gpu), requires_grad=False))
    residual.lsh_residual_norm_fwd(cfg, x, f, None, weights)
    weights.post_g.data = weights.post_g.data.to(BF)
    with pytest.raises(ValueError, match="dtype"):
        residual.lsh_residual_norm_fwd(cfg, x, f, None, weights)
