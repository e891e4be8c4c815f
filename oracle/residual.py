"""fp64 oracle of the step between two blocks (NumPy): forward, backward, and how far fp32 arithmetic may be off."""
from __future__ import annotations

import numpy as np

E = 2.0 ** -24  # half an fp32 step
SUM = 40  # additions on the way of a row's sum: 8 in a thread, 6 over a wave, up to 16 waves, and the products' own


def sigmoid(x):
    return np.where(x >= 0, 1 / (1 + np.exp(-np.abs(x))), np.exp(-np.abs(x)) / (1 + np.exp(-np.abs(x))))


class Norm:
    """A row's norm: n, r = 1 / deviation, and bounds dn of |n|'s and dr of r's relative error in fp32, for rows that are
    themselves off by dt."""

    def __init__(self, t, layer, eps, dt=0.0):
        mean = t.mean(-1, keepdims=True) if layer else 0.0
        d = t - mean
        ms = (d * d).mean(-1, keepdims=True) + eps
        self.r = np.where(ms > 0, 1 / np.sqrt(np.where(ms > 0, ms, 1)), 0.0)
        self.n, self.layer = d * self.r, layer
        dmean = 0.0
        if layer:
            dmean = SUM * E * np.abs(t).mean(-1, keepdims=True) + (np.mean(dt, -1, keepdims=True) if np.ndim(dt) else dt)
        dd = dmean + dt + E * np.abs(d)
        # the mean square: its own sum, and what its terms are off by
        off = SUM * E + 2 * (np.abs(self.n) * dd * self.r).mean(-1, keepdims=True) + (dd * self.r).max(-1, keepdims=True) ** 2
        self.dr = off / 2 * 1.1 + 4 * E
        self.dn = dd * self.r * (1 + self.dr) + np.abs(self.n) * (self.dr + E)

    def back(self, d, dd):
        """norm'(d) and the bound of its error, for d off by dd."""
        n, r = self.n, self.r
        s, ds = (d * n).mean(-1, keepdims=True), (np.abs(d) * self.dn + dd * np.abs(n) + (SUM + 2) * E * np.abs(d * n)).mean(-1, keepdims=True)
        t, dt = (d.mean(-1, keepdims=True), (dd + SUM * E * np.abs(d)).mean(-1, keepdims=True)) if self.layer else (0.0, 0.0)
        inner = d - t - n * s
        size = np.abs(d) + np.abs(t) + np.abs(n * s)
        return r * inner, r * (dd + dt + np.abs(n) * ds + self.dn * np.abs(s) + 3 * E * size) * (1 + self.dr) + r * np.abs(inner) * (self.dr + E)


def _branch(c, f, gate, w):
    """u, its bound, gate', its slope, and f's Norm."""
    norm, u, du = None, f, 0.0
    if c["post"]:
        norm = Norm(f, c["layer"], c["eps"])
        b = 0.0 if w["post_b"] is None else w["post_b"]
        u = norm.n * w["post_g"] + b
        du = np.abs(w["post_g"]) * norm.dn + E * np.abs(u)
    if c["gate"] == "sigmoid":
        g = sigmoid(gate)
        return u, du, g, g * sigmoid(-gate), norm
    return u, du, (gate if c["gate"] == "linear" else np.ones_like(f)), np.ones_like(f), norm


def forward(c, x, f, gate, w):
    """{"y", "z"} and the bounds {"y", "z"} of their errors before any rounding to 16 bits."""
    x = np.zeros_like(f) if x is None else x
    y, dy = x, np.zeros_like(x)
    if f is not None:
        u, du, g, _, _ = _branch(c, f, gate, w)
        m = c["alpha"] * (1.0 if w["scale"] is None else w["scale"]) * g
        y = x + m * u
        dy = np.abs(m) * du + 12 * E * np.abs(m * u) + E * np.abs(y)  # exp, sum, quotient and two products in m
    out, tol = {"y": y}, {"y": dy}
    if c["pre"]:
        norm = Norm(y, c["layer"], c["eps"], dy)
        b = 0.0 if w["pre_b"] is None else w["pre_b"]
        out["z"] = norm.n * w["pre_g"] + b
        tol["z"] = np.abs(w["pre_g"]) * norm.dn + E * np.abs(out["z"])
    return out, tol


def backward(c, y, f, gate, w, dy, dz):
    """The gradients and the bounds of their errors, both by name."""
    out, tol = {}, {}
    rows = len(dz if dy is None else dy)

    def column(name, terms, off):
        out[name], tol[name] = terms.sum(0), off.sum(0) + (rows + 20) * E * np.abs(terms).sum(0)

    dx, ddx = (0.0, 0.0) if dy is None else (dy, 0.0)
    if c["pre"]:
        norm = Norm(y, c["layer"], c["eps"])
        column("dpre_g", dz * norm.n, np.abs(dz) * norm.dn)
        if w["pre_b"] is not None:
            column("dpre_b", dz, 0 * dz)
        d = dz * w["pre_g"]
        more, off = norm.back(d, E * np.abs(d))
        dx, ddx = dx + more, off + E * np.abs(dx + more)
    out["dx"], tol["dx"] = dx, ddx + 0 * dx
    if f is None:
        return out, tol
    u, du, g, slope, norm = _branch(c, f, gate, w)
    a = c["alpha"] * (1.0 if w["scale"] is None else w["scale"]) * np.ones_like(f)
    dm, ddm = dx * u, np.abs(dx) * du + ddx * np.abs(u) + E * np.abs(dx * u)
    if gate is not None:
        out["dgate"] = dm * a * slope
        tol["dgate"] = ddm * np.abs(a * slope) + 14 * E * np.abs(out["dgate"])
    if w["scale"] is not None:
        column("dscale", dm * c["alpha"] * g, (ddm + 14 * E * np.abs(dm)) * np.abs(c["alpha"] * g))
    d = dx * a * g
    dd = (ddx + 14 * E * np.abs(dx)) * np.abs(a * g)
    if norm is not None:
        column("dpost_g", d * norm.n, dd * np.abs(norm.n) + np.abs(d) * norm.dn)
        if w["post_b"] is not None:
            column("dpost_b", d, dd)
        d, dd = d * w["post_g"], (dd + E * np.abs(d)) * np.abs(w["post_g"])
        d, dd = norm.back(d, dd)
    out["df"], tol["df"] = d, dd
    return out, tol
