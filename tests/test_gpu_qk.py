"""GPU parity of the per-head norm with rotation, forward and backward, with the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import qk as Q
from paper_2001_04451_amd import qk

from gpu_common import log

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    qk.lib()
    return torch.device("cuda:0")


def freqs(rot, base=10000.0):
    return (base ** (-np.arange(rot // 2) * 2.0 / max(rot, 1))).astype(np.float32)


class Case:
    def __init__(self, dtype, T, Hq, Hk=0, L=0, rot=64, inter=False, per_head=False, pos="none", eps=1e-6, seed=0, wide=0):
        rng = np.random.default_rng(seed)
        self.dtype, self.T, self.Hq, self.Hk, self.L = dtype, T, Hq, Hk, L
        H = Hq + Hk
        x = rng.standard_normal((T, H * 64 + wide)) * np.exp(rng.standard_normal((T, 1)))
        self.x = torch.from_numpy(x.astype(np.float32)).to(dtype)
        self.g = (1 + 0.3 * rng.standard_normal((H, 64) if per_head else (2, 64))).astype(np.float32)
        self.freq = freqs(rot)
        self.pos = {"none": None, "near": np.arange(T) % 77, "far": rng.integers(1 << 20, 1 << 24, T),
                    "any": rng.integers(-2 ** 31, 2 ** 31, T)}[pos]
        self.cfg = qk.QkConfig(T=T, Hq=Hq, Hk=Hk, L=L, rot=rot, interleaved=inter, gain_per_head=per_head, eps=eps)
        self.dq, self.dk = (rng.standard_normal(self.cfg.out_shape(h)).astype(np.float32) if h else None for h in (Hq, Hk))

    def gains(self, gpu):
        gq, gk = (self.g[:self.Hq], self.g[self.Hq:]) if self.cfg.gain_per_head else (self.g[0], self.g[1])
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(gpu)
        return up(gq), up(gk) if self.Hk else None

    def args(self, gpu):
        gq, gk = self.gains(gpu)
        pos = None if self.pos is None else torch.from_numpy(self.pos.astype(np.int32)).to(gpu)
        return self.x.to(gpu), gq, gk, torch.from_numpy(self.freq).to(gpu), pos

    def parts(self):
        """(heads of x, gain, upstream gradient) in fp64 for queries and keys."""
        H = self.Hq + self.Hk
        x = self.x.double().numpy()[:, :H * 64].reshape(self.T, H, 64)
        for i, (a, b, d) in enumerate(((0, self.Hq, self.dq), (self.Hq, H, self.dk))):
            if a < b:
                g = self.g[a:b] if self.cfg.gain_per_head else self.g[i]
                yield x[:, a:b], g.astype(np.float64), Q.tokens_first(d) if self.L else d

    def ref_args(self):
        pos = self.pos if self.pos is not None else (np.arange(self.T) % self.L if self.L else np.arange(self.T))
        return pos, self.freq.astype(np.float64), self.cfg.rot, self.cfg.interleaved, self.cfg.eps


# fp32 roundings: the mean square (at most 66 half steps under a root), root, quotient, x r g, cos and sin (2 half steps
# of one, the angle's reduction 2^-24 turns and for positions past 2^29 the product's rounding), two products and a sum
EPS = 2.0 ** -24


def turn_error(c):
    far = 0 if c.pos is None else np.abs(np.asarray(c.pos, np.float64)).max()
    return 2 * np.pi * (EPS + far * 2.0 ** -53) + 4 * EPS


def check_forward(c, gpu):
    q, k = qk.lsh_qk_norm_rotate_fwd(c.cfg, *c.args(gpu))
    torch.cuda.synchronize()
    assert (k is None) == (c.Hk == 0)
    for got, (x, g, _) in zip((q, k), c.parts()):
        ref = Q.norm_rotate(x, g, *c.ref_args())
        pair = np.abs(Q.norm_rotate(x, g, c.ref_args()[0], c.ref_args()[1][:0], 0, False, c.cfg.eps))
        a, b = Q._pairs(c.cfg.rot, c.cfg.interleaved)
        size = pair.copy()  # |a| + |b| of the element's pair
        size[..., a] = size[..., b] = pair[..., a] + pair[..., b]
        tol = size * ((33 + 8) * EPS + turn_error(c)) + np.abs(ref) * (torch.finfo(c.dtype).eps / 2) * 1.001
        got = got.double().cpu().numpy()
        err = np.abs((Q.tokens_first(got) if c.L else got) - ref)
        assert (err <= tol).all(), f"off by {err.max():.3e}, {(err / np.maximum(tol, 1e-300)).max():.2f} of the tolerance"
    return q, k


def check_backward(c, gpu):
    up = lambda a: None if a is None else torch.from_numpy(a).to(gpu)
    H = c.Hq + c.Hk
    dx, dgq, dgk = qk.lsh_qk_norm_rotate_bwd(c.cfg, *c.args(gpu), up(c.dq), up(c.dk))
    torch.cuda.synchronize()
    got_dx = dx.double().cpu().numpy().reshape(c.T, H, 64)
    h0 = 0
    for got_g, (x, g, d) in zip((dgq, dgk), c.parts()):
        ref, dg, dg_abs = Q.norm_rotate_bwd(x, g, *c.ref_args(), d)
        n = x.shape[1]
        ms = (x * x).mean(-1, keepdims=True) + c.cfg.eps
        r = np.where(ms > 0, 1 / np.sqrt(np.where(ms > 0, ms, 1)), 0)
        # a gradient's turned pair is at most |u| <= sqrt(2) max |d| a value; w and the mean of w n likewise, |n| <= 8
        size = r * (np.abs(g).max() * np.abs(d).max(-1, keepdims=True) * 2 * (1 + np.abs(x * r) * np.abs(x * r).mean(-1, keepdims=True)))
        tol = size * ((33 + 16 + 66) * EPS + turn_error(c))
        err = np.abs(got_dx[:, h0:h0 + n] - ref)
        assert (err <= tol).all(), f"dx off by {err.max():.3e}, {(err / np.maximum(tol, 1e-300)).max():.2f} of the tolerance"
        # the gain's sum: at most (tokens and heads of a workgroup) + 40 fp32 additions of terms whose magnitudes sum to
        # dg_abs (a term's own error counts its pair's size, at most 3 times the mean term over these Gaussian rows)
        adds = -(-c.T // min(1024, -(-c.T // 16))) * n + 40
        gtol = dg_abs * ((adds + 60) * EPS + 3 * turn_error(c)) + 2 * EPS * np.abs(dg)
        gerr = np.abs(got_g.double().cpu().numpy() - dg)
        assert (gerr <= gtol).all(), f"dgain off by {gerr.max():.3e}, {(gerr / gtol).max():.2f} of the tolerance"
        h0 += n
    return dx, dgq, dgk


SHAPES = [dict(T=1, Hq=1), dict(T=1, Hq=3, Hk=1, L=1), dict(T=7, Hq=16), dict(T=130, Hq=6, Hk=2, L=65),
          dict(T=1001, Hq=12, Hk=3), dict(T=33, Hq=40, Hk=5, L=11), dict(T=4096, Hq=2, L=1024), dict(T=17, Hq=1, Hk=1)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("per_head", [False, True])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_norm_rotate(gpu, dtype, inter, per_head, shape):
    kw = SHAPES[shape]
    c = Case(dtype, **kw, inter=inter, per_head=per_head, rot=(64, 16, 32, 48, 64, 64, 32, 48)[shape],
             pos=("near", "none", "far", "none", "far", "near", "none", "any")[shape], seed=shape)
    log("norm rotate", dtype, inter, per_head, kw)
    check_forward(c, gpu)
    check_backward(c, gpu)


def test_no_rotation_and_zero_rows(gpu):
    """rot = 0 needs no frequencies' values; zero rows give zeros with eps = 0 and finite gradients."""
    c = Case(torch.float32, 9, 2, 1, rot=0, eps=0.0)
    c.x[4] = 0
    log("norm rotate zero rows")
    q, k = check_forward(c, gpu)
    assert not q[4].any() and not k[4].any()
    dx, _, _ = check_backward(c, gpu)
    assert not dx[4].any()
    c = Case(torch.bfloat16, 9, 2, 1, eps=1e-6)
    c.x[4] = 0
    check_forward(c, gpu)
    check_backward(c, gpu)


def test_large_and_small_rows(gpu):
    c = Case(torch.float32, 6, 2, eps=0.0)
    c.x *= torch.tensor([2.0 ** e for e in (-59, -30, 0, 20, 50, 55)])[:, None]
    log("norm rotate sizes")
    check_forward(c, gpu)


def test_strided_rows_stay_inside(gpu):
    """x and dx as views of wider rows: nothing beside them is read into the result or written; the same bits as packed."""
    c = Case(torch.bfloat16, 50, 2, 1, wide=72)
    packed = Case(torch.bfloat16, 50, 2, 1)
    packed.x, packed.g, packed.dq, packed.dk = c.x[:, :192].contiguous(), c.g, c.dq, c.dk
    x, gq, gk, freq, pos = c.args(gpu)
    x[:, 192:] = float("nan")
    up = lambda a: torch.from_numpy(a).to(gpu)
    log("norm rotate strided")
    q, k = qk.lsh_qk_norm_rotate_fwd(c.cfg, x, gq, gk, freq)
    pq, pk = check_forward(packed, gpu)
    assert torch.equal(q, pq) and torch.equal(k, pk)
    dx = torch.full((50, 200), 7.0, device=gpu)
    qk.lsh_qk_norm_rotate_bwd(c.cfg, x, gq, gk, freq, None, up(c.dq), up(c.dk), dx=dx)
    pdx, _, _ = check_backward(packed, gpu)
    assert torch.equal(dx[:, :192], pdx) and (dx[:, 192:] == 7).all()


def test_repeats_bit_for_bit_on_a_side_stream_and_in_a_graph(gpu):
    c = Case(torch.bfloat16, 3000, 4, 2, L=1000, per_head=False, pos="near")
    args = c.args(gpu)
    dq, dk = (torch.from_numpy(a).to(gpu) for a in (c.dq, c.dk))
    want = check_forward(c, gpu) + check_backward(c, gpu)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    log("norm rotate stream and graph")
    with torch.cuda.stream(side):
        got = qk.lsh_qk_norm_rotate_fwd(c.cfg, *args) + qk.lsh_qk_norm_rotate_bwd(c.cfg, *args, dq, dk)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    outs = [torch.empty_like(t) for t in want]
    ws = torch.empty(qk.qk_workspace_bytes(c.cfg), dtype=torch.uint8, device=gpu)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        qk.lsh_qk_norm_rotate_fwd(c.cfg, *args, q=outs[0], k=outs[1])
        qk.lsh_qk_norm_rotate_bwd(c.cfg, *args, dq, dk, dx=outs[2], dgain_q=outs[3], dgain_k=outs[4], workspace=ws)
    for i in range(3):
        for t in outs:
            t.fill_(float("nan"))
        ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs)), i
        args[0].mul_(-1 if i else 1)  # the next replay on other rows, against eager
        want = qk.lsh_qk_norm_rotate_fwd(c.cfg, *args) + qk.lsh_qk_norm_rotate_bwd(c.cfg, *args, dq, dk)


def test_binding_refusals(gpu):
    c = Case(torch.bfloat16, 6, 2, 1)
    x, gq, gk, freq, pos = c.args(gpu)
    with pytest.raises(ValueError, match="gain_k"):
        qk.lsh_qk_norm_rotate_fwd(c.cfg, x, gq, None, freq)
    with pytest.raises(ValueError, match="shape"):
        qk.lsh_qk_norm_rotate_fwd(c.cfg, x[:, :128], gq, gk, freq)
    with pytest.raises(ValueError, match="contiguous"):
        qk.lsh_qk_norm_rotate_fwd(c.cfg, x.t().contiguous().t(), gq, gk, freq)
    with pytest.raises(ValueError, match="dtype"):
        qk.lsh_qk_norm_rotate_fwd(c.cfg, x, gq.bfloat16(), gk, freq)
    with pytest.raises(TypeError):
        qk.lsh_qk_norm_rotate_fwd(c.cfg, x.half(), gq, gk, freq)
    with pytest.raises(ValueError, match="freq"):
        qk.lsh_qk_norm_rotate_fwd(c.cfg, x, gq, gk, freq[:8])
    with pytest.raises(ValueError, match="dk is required"):
        qk.lsh_qk_norm_rotate_bwd(c.cfg, x, gq, gk, freq, None, torch.zeros(6, 2, 64, device=gpu))
