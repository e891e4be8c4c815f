"""The oracles of the 4-bit weights and of the step between two blocks against other formulations, on the CPU."""
import numpy as np
import pytest
import torch

from oracle import residual as R
from oracle import w4 as W


@pytest.mark.parametrize("type_,group,zeros", [("int4", 32, False), ("int4", 64, True), ("int4", 128, True), ("e2m1", 32, False)])
def test_quantised_values_are_the_nearest(type_, group, zeros):
    """No value is further from its own than half a step of its group, and no smaller scale would hold the group."""
    rng = np.random.default_rng(3)
    w = rng.standard_normal((5, 160)) * np.exp(rng.standard_normal((5, 1)))
    w[1, :group] = 0
    w[2, :group] = 3.5
    w = w.astype(np.float32).astype(np.float64)
    codes, scales, zps = W.quantize(w, type_, group, zeros)
    back = W.values(codes, scales, zps, type_, group)
    every = W.bf16_values()
    for n in range(5):
        for g in range(-(-160 // group)):
            x, y, c = (t[n, g * group:(g + 1) * group] for t in (w, back, codes))
            s = 2.0 ** (int(scales[n, g]) - 127) if type_ == "e2m1" else every[scales[n, g]]
            if not x.any():
                assert not y.any()
                continue
            step = s * np.where(np.abs(x) > 4 * s, 2, np.where(np.abs(x) > 2 * s, 1, 0.5)) if type_ == "e2m1" else s
            # the zero point's own rounding moves the ends of the range by up to half a step, where 15 cuts off
            assert (np.abs(x - y) <= step / 2 * (1 + 1e-12) + (s / 2 if zeros else 0)).all()
            span = max(0, x.max()) - min(0, x.min()) if zeros else np.abs(x).max()
            most = 15 if zeros else 7 if type_ == "int4" else 6
            smaller = s / 2 if type_ == "e2m1" else every[scales[n, g] - 1]
            assert most * s >= span > most * smaller
            assert c.max() <= 15


def test_e2m1_codes_are_those_of_the_cache():
    from oracle import cache as C
    rng = np.random.default_rng(4)
    w = (rng.standard_normal((7, 64)) * 10.0 ** rng.integers(-3, 4, (7, 1))).astype(np.float32)
    w[0, :8] = [2.5, 3.5, 5.0, 0.25, 0.75, -2.5, 6.0, -0.0]
    codes, scales, _ = W.quantize(w, "e2m1", 32, False)
    cc, cs = C.encode(w, "e2m1")
    assert np.array_equal(W.pack_rows(codes), cc) and np.array_equal(scales, cs)


def _case(layer, gate, post, pre, bias, scale, T=5, D=16, seed=0):
    rng = np.random.default_rng(seed)
    c = dict(layer=layer, gate=gate, post=post, pre=pre, eps=1e-5, alpha=-0.7)
    a = lambda *s: rng.standard_normal(s)
    w = dict(scale=1 + 0.2 * a(D) if scale else None)
    for n, on in (("post", post), ("pre", pre)):
        w[n + "_g"] = 1 + 0.2 * a(D) if on else None
        w[n + "_b"] = a(D) if on and bias else None
    return c, a(T, D) + 0.5, a(T, D) + 0.2, a(T, D) if gate != "none" else None, w, a(T, D), a(T, D) if pre else None


CASES = [(layer, gate, post, pre, bias, scale) for layer in (False, True) for gate in ("none", "linear", "sigmoid")
         for post, pre in ((True, True), (True, False), (False, True)) for bias, scale in ((True, True), (False, False))]


@pytest.mark.parametrize("case", CASES)
def test_residual_oracle_against_autograd(case):
    """Forward and backward of the definition, by torch's own layer norm and autograd in fp64."""
    c, x, f, gate, w, dy, dz = _case(*case)
    t = lambda v: None if v is None else torch.from_numpy(v).requires_grad_()
    X, F, G = t(x), t(f), t(gate)
    P = {n: t(v) for n, v in w.items()}

    def norm(v, which):
        if c["layer"]:
            n = torch.nn.functional.layer_norm(v, v.shape[-1:], eps=c["eps"])
        else:
            n = v / (v.pow(2).mean(-1, keepdim=True) + c["eps"]).sqrt()
        n = n * P[which + "_g"]
        return n if P[which + "_b"] is None else n + P[which + "_b"]

    u = norm(F, "post") if c["post"] else F
    g = 1.0 if G is None else torch.sigmoid(G) if c["gate"] == "sigmoid" else G
    y = X + c["alpha"] * g * u * (1.0 if P["scale"] is None else P["scale"])
    y.retain_grad()
    loss = (y * torch.from_numpy(dy)).sum()
    if c["pre"]:
        z = norm(y, "pre")
        loss = loss + (z * torch.from_numpy(dz)).sum()
    loss.backward()
    out, tol = R.forward(c, x, f, gate, w)
    assert np.allclose(out["y"], y.detach().numpy(), rtol=1e-13, atol=1e-13)
    if c["pre"]:
        assert np.allclose(out["z"], z.detach().numpy(), rtol=1e-12, atol=1e-13)
    grads, gtol = R.backward(c, out["y"], f, gate, w, dy, dz)
    want = {"dx": X, "df": F, "dgate": G, **{"d" + n: v for n, v in P.items()}}
    assert set(grads) == {n for n, v in want.items() if v is not None}
    for n in grads:
        assert np.allclose(grads[n], want[n].grad.numpy(), rtol=1e-11, atol=1e-12), n
        assert (gtol[n] >= 0).all() and (gtol[n] < 1e-3 * (1 + np.abs(grads[n]).max())).all()


def test_residual_oracle_against_differences():
    c, x, f, gate, w, dy, dz = _case(True, "sigmoid", True, True, True, True, T=2, D=8)

    def loss(**kw):
        v = dict(x=x, f=f, gate=gate, **w)
        v.update(kw)
        out, _ = R.forward(c, v["x"], v["f"], v["gate"], {n: v[n] for n in w})
        return (out["y"] * dy).sum() + (out["z"] * dz).sum()

    y = R.forward(c, x, f, gate, w)[0]["y"]
    grads, _ = R.backward(c, y, f, gate, w, dy, dz)
    for name, base in (("x", x), ("f", f), ("gate", gate), *w.items()):
        g, h = grads["d" + name], 1e-6
        for i in np.ndindex(base.shape):
            up, down = base.copy(), base.copy()
            up[i] += h
            down[i] -= h
            assert abs((loss(**{name: up}) - loss(**{name: down})) / (2 * h) - g[i]) < 1e-7 * (1 + abs(g[i])), (name, i)


def test_a_row_without_deviation():
    """eps = 0: such rows are 0 and their gradient is 0."""
    c = dict(layer=True, gate="none", post=True, pre=True, eps=0.0, alpha=1.0)
    w = dict(scale=None, post_g=np.ones(8), post_b=None, pre_g=np.ones(8), pre_b=None)
    f, x = np.full((1, 8), 2.0), np.zeros((1, 8))
    out, _ = R.forward(c, x, f, None, w)
    assert not out["y"].any() and not out["z"].any()
    grads, _ = R.backward(c, out["y"], f, None, w, np.zeros((1, 8)), np.ones((1, 8)))
    assert not grads["dx"].any() and not grads["df"].any()
