"""The work of a decoding layer around the cache's attention, and of the norms between layers in training.

``listed()`` names the cases, ``draw()`` gives others of the same ranges, ``prepare`` makes what a program
holds before the call, ``run`` is one pass (elementary torch, or with ``own`` the library's calls), ``work``
the bytes and operations a pass cannot do without, ``exact`` the outputs in 64 bits.

Kinds of case:
  linear    rows times a matrix held in 4 bits with a scale for each group of inputs;
  quantise  a matrix into that form, and its values back;
  append    projected rows, normed per head and rotated to their positions: queries out, keys and values into
            the paged cache (whose new rows are read back);
  residual  a block's output normed, gated and added to the residual stream, and the stream normed for the next
            block; with ``train`` the backward too.
"""
import math
import random

import torch

own = False

D = 64  # head width
BLOCK = 32  # values that share a power-of-two scale
EPS = 1e-6
CODES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)  # e2m1 magnitudes, by their codes
BITS = {"e4m3": (3, -6, 0.875, 9), "e2m1": (1, 0, 0.75, 3)}  # mantissa bits, lowest exponent, largest = m 2^e


def listed():
    return [
        # the smallest product: one sequence's next token through a feed-forward layer's first product
        dict(name="linear_one_4096x1024", kind="linear", type="int4", group=128, zeros=False, M=1, N=4096, K=1024,
             bias=True, out="relu"),
        # one token's scores over a vocabulary, the largest matrix of a step
        dict(name="linear_one_32000x4096", kind="linear", type="e2m1", group=32, zeros=False, M=1, N=32000, K=4096,
             bias=False, out="f32"),
        # a serving batch's second product onto the residual stream, zero points, small groups
        dict(name="linear_16_4096x4096_zeros", kind="linear", type="int4", group=64, zeros=True, M=16, N=4096, K=4096,
             bias=True, out="resid"),
        # a ragged batch, an odd number of outputs and a last group that is cut short
        dict(name="linear_61_odd", kind="linear", type="int4", group=128, zeros=True, M=61, N=2047, K=4128, bias=False,
             out="f32"),
        # a prompt through the same matrix as the first case
        dict(name="linear_prompt_2k", kind="linear", type="int4", group=128, zeros=False, M=2048, N=4096, K=1024,
             bias=True, out="relu"),
        # weights as they are loaded: a feed-forward matrix in bf16, and a wide one in fp32
        dict(name="quantise_4096x1024_e2m1", kind="quantise", type="e2m1", group=32, zeros=False, dtype="bf16", N=4096,
             K=1024),
        dict(name="quantise_16384x4096_int4", kind="quantise", type="int4", group=128, zeros=True, dtype="f32", N=16384,
             K=4096),
        # a decoding step's projected rows: 64 sequences of 16 heads with shared keys, e4m3
        dict(name="append_decode_64", kind="append", dtype="bf16", type="e4m3", n_seq=64, new=1, H=16, Hkv=16, len=8000,
             ragged=True, page=64, shared=True, norm=True, rot=64, inter=False, per_head=False),
        # prompts of several sequences with grouped heads into a 4-bit cache, fp32 rows, half the width rotated
        dict(name="append_prompts_grouped_e2m1", kind="append", dtype="f32", type="e2m1", n_seq=5, new=3277, H=16,
             Hkv=4, len=9001, ragged=True, page=32, shared=False, norm=False, rot=32, inter=True, per_head=False),
        # one decoding step's rows between two layers
        dict(name="residual_decode_16", kind="residual", dtype="bf16", T=16, D=4096, norm="rms", pre=True, post=True,
             gate="none", scale=True, bias=False, train=False),
        # fine-tuning on ragged rows of an odd width, layer norms with biases, a gate for every value
        dict(name="residual_f32_ragged_train", kind="residual", dtype="f32", T=5997, D=1000, norm="layer", pre=True,
             post=True, gate="sigmoid", scale=True, bias=True, train=True),
        # the reversible block's training batch: 65,536 rows of 1024
        dict(name="residual_64k_train", kind="residual", dtype="bf16", T=65536, D=1024, norm="rms", pre=True, post=True,
             gate="sigmoid", scale=False, bias=False, train=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear", "quantise", "append", "append", "residual", "residual"])
    if kind in ("linear", "quantise"):
        type_ = rng.choice(["int4", "int4", "e2m1"])
        group, zeros = (rng.choice([32, 64, 128, 128]), rng.random() < 0.5) if type_ == "int4" else (32, False)
        K = 32 * _log(rng, 2, 512)
        most = 32000 * 4096 if kind == "linear" else 16384 * 4096
        N = _log(rng, 16, min(32000, most // K))
        N = N if rng.random() < 0.4 else -(-N // 16) * 16
        c = dict(kind=kind, type=type_, group=group, zeros=zeros, N=N, K=K)
        if kind == "quantise":
            return dict(c, dtype=rng.choice(["bf16", "f32"]))
        most = max(1, min(2048, (1 << 33) // (N * K)))
        M = 1 if rng.random() < 0.25 else _log(rng, 1, most)
        return dict(c, M=M, bias=rng.random() < 0.5, out=rng.choice(["relu", "bf16", "f32", "resid"]))
    if kind == "append":
        shared = rng.random() < 0.5
        H = rng.choice([1, 2, 4, 8, 8, 16, 16])
        new = 1 if rng.random() < 0.4 else _log(rng, 1, 16384)
        n_seq = _log(rng, 1, max(1, min(128, 16384 // new)))
        return dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f32"]), type=rng.choice(["bf16", "e4m3", "e2m1"]),
                    n_seq=n_seq, new=new, H=H, Hkv=H if shared else rng.choice([h for h in (1, 2, 4, 8) if H % h == 0]),
                    len=new + _log(rng, 1, max(1, min(8192, (1 << 18) // n_seq))), ragged=rng.random() < 0.5,
                    page=rng.choice([16, 32, 64, 64, 128, 256]), shared=shared, norm=rng.random() < 0.6,
                    rot=rng.choice([64, 64, 32, 16, 48]), inter=rng.random() < 0.5, per_head=rng.random() < 0.4)
    width = 8 * _log(rng, 8, 1024)
    T = _log(rng, 1, min(65536, (1 << 26) // width))
    pre = rng.random() < 0.85
    return dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f32"]), T=T, D=width, norm=rng.choice(["rms", "layer"]),
                pre=pre, post=not pre or rng.random() < 0.6, gate=rng.choice(["none", "linear", "sigmoid"]),
                scale=rng.random() < 0.5, bias=rng.random() < 0.5, train=rng.random() < 0.5)


# ----------------------------------------------------------------------------
# inputs


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return {"linear": _prepare_linear, "quantise": _prepare_quantise, "append": _prepare_append,
            "residual": _prepare_residual}[case["kind"]](case, g)


def _weights(c, g):
    """A matrix as training leaves it: outputs of unequal size, a few large values."""
    w = _randn(g, c["N"], c["K"]) * torch.exp(0.3 * _randn(g, c["N"], 1)) / math.sqrt(c["K"])
    return w * (1 + 3 * (_randn(g, c["N"], c["K"]).abs() > 3.5))


def _w4_config(c):
    from paper_2001_04451_amd import w4
    return w4.W4Config(N=c["N"], K=c["K"], type=c["type"], group=c["group"], zeros=c["zeros"])


def _prepare_linear(c, g):
    s = {"c": c}
    codes, s["scale"], s["zero"] = _to_codes(c, _weights(c, g))
    s["codes"] = codes[:, 0::2] | (codes[:, 1::2] << 4)  # two a byte, the even input in the low half
    s["a"] = (_randn(g, c["M"], c["K"]) * torch.exp(0.5 * _randn(g, c["K"]))).to(torch.bfloat16)
    s["bias"] = 0.1 * _randn(g, c["N"]) if c["bias"] else None
    s["resid"] = _randn(g, c["M"], c["N"]) if c["out"] == "resid" else None
    if own:
        from paper_2001_04451_amd import w4
        s["cfg"] = _w4_config(c)
        s["packed"] = w4.lsh_w4_pack(s["cfg"], s["codes"], s["scale"], s["zero"])
        s["workspace"] = w4.workspace(s["cfg"], c["M"], s["a"].device)
    return s


def _prepare_quantise(c, g):
    s = {"c": c, "w": _weights(c, g).to(_dtype(c))}
    if own:
        s["cfg"] = _w4_config(c)
    return s


def _counts(c):
    """New tokens and cached length of each sequence; from the case alone."""
    n = c["n_seq"]
    lens = [c["len"]] * n
    if c["ragged"]:  # spread over the length's logarithm, down to a thirty-second, in a fixed disorder
        lens = [max(1, int(round(c["len"] * 32.0 ** (-i / max(1, n - 1))))) for i in range(n)]
        random.Random(n * 1000003 + c["len"]).shuffle(lens)
    return [min(c["new"], m) for m in lens], lens


def _prepare_append(c, g):
    news, lens = _counts(c)
    H, Hkv, page, rot = c["H"], c["Hkv"], c["page"], c["rot"]
    Hk, T, n_seq = 0 if c["shared"] else Hkv, sum(news), len(news)
    used = [-(-n // page) for n in lens]
    n_pages, most = sum(used) + 3, max(used)
    where = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    start = torch.tensor([sum(used[:i]) for i in range(n_seq)], device="cuda")[:, None]
    col, count = torch.arange(most, device="cuda")[None], torch.tensor(used, device="cuda")[:, None]
    table = torch.where(col < count, where[(start + col).clamp(max=n_pages - 1)], -1).to(torch.int32)
    s = {"c": c, "news": news, "table": table, "len": torch.tensor(lens, dtype=torch.int32, device="cuda"),
         "first": torch.tensor([sum(news[:i]) for i in range(n_seq + 1)], dtype=torch.int32, device="cuda")}
    size = torch.exp(0.5 * _randn(g, (H + Hk + Hkv) * D))  # channels of unequal size, as a projection gives them
    s["x"] = (_randn(g, T, (H + Hk + Hkv) * D) * size).to(_dtype(c))
    s["gq"] = s["gk"] = None
    if c["norm"]:
        s["gq"] = 1 + 0.1 * _randn(g, *((H, D) if c["per_head"] else (D,)))
        s["gk"] = 1 + 0.1 * _randn(g, *((Hk, D) if c["per_head"] else (D,))) if Hk else None
    s["freq"] = (10000.0 ** (-torch.arange(rot // 2, device="cuda", dtype=torch.float64) * 2 / rot)).float()
    # the pool: what lies in it before the step does not matter here, only which slots the step writes
    slots, row = (n_pages, Hkv, page), {"bf16": 2 * D, "e4m3": D, "e2m1": D // 2}[c["type"]]
    scaled = c["type"] != "bf16"
    for name, shape, dt, there in (("k", slots + (row,), torch.uint8, True), ("v", slots + (row,), torch.uint8, True),
                                   ("k_scale", slots + (2,), torch.uint8, scaled),
                                   ("v_scale", slots + (2,), torch.uint8, scaled),
                                   ("k_inv", slots, torch.float32, c["shared"])):
        s[name] = torch.zeros(shape, dtype=dt, device="cuda") if there else None
    if own:
        from paper_2001_04451_amd import cache, qk
        s["cfg"] = cache.CacheConfig(n_seq=n_seq, T=T, H=H, Hkv=Hkv, n_pages=n_pages, max_pages=most, page=page,
                                     type=c["type"], shared_qk=c["shared"], max_new=max(news))
        s["qk"] = qk.QkConfig(T=T, Hq=H, Hk=Hk, rot=rot, interleaved=c["inter"], gain_per_head=c["per_head"], eps=EPS)
        s["pages"] = cache.Pages(k=s["k"], v=s["v"], k_scale=s["k_scale"], v_scale=s["v_scale"], k_inv=s["k_inv"])
        s["seqs"] = cache.Sequences(first=s["first"], length=s["len"], table=s["table"])
    return s


def _prepare_residual(c, g):
    T, W, dt = c["T"], c["D"], _dtype(c)
    s = {"c": c, "x": 2 * _randn(g, T, W) + 0.3, "f": (_randn(g, T, W) * torch.exp(0.5 * _randn(g, W)) + 0.1).to(dt)}
    s["gate"] = _randn(g, T, W).to(dt) if c["gate"] != "none" else None
    s["scale"] = 0.5 + 0.1 * _randn(g, W) if c["scale"] else None
    for name in ("post", "pre"):
        s[name + "_g"] = 1 + 0.1 * _randn(g, W) if c[name] else None
        s[name + "_b"] = 0.1 * _randn(g, W) if c[name] and c["bias"] else None
    if c["train"]:
        s["dy"] = _randn(g, T, W)
        s["dz"] = _randn(g, T, W) if c["pre"] else None
    if own:
        from paper_2001_04451_amd import residual
        s["cfg"] = residual.ResidualConfig(T=T, D=W, norm=c["norm"], pre=c["pre"], post=c["post"], gate=c["gate"],
                                           eps=EPS)
        s["weights"] = residual.ResidualWeights(scale=s["scale"], post_g=s["post_g"], post_b=s["post_b"],
                                                pre_g=s["pre_g"], pre_b=s["pre_b"])
    return s


# ----------------------------------------------------------------------------
# the plain forms


def _to_codes(c, w):
    """Codes [N][K], scales [N][groups] and zero points (or None) of a matrix: the smallest scale (a bf16 value, or
    for e2m1 a power of two as its exponent + 127) under which the group's values fit the codes' range, and the
    nearest code, ties to even.  In 64 bits, for values next to a border."""
    N, K, G = c["N"], c["K"], c["group"]
    groups = -(-K // G)
    x = torch.nn.functional.pad(w.float(), (0, groups * G - K)).view(N, groups, G)
    if c["type"] == "e2m1":
        m, e = torch.frexp(x.abs().amax(-1, keepdim=True))
        e = torch.where(m == 0, -127, e - 3 + (m > 0.75).to(e.dtype)).clamp(-127, 127)
        y = torch.ldexp(x.double(), -e).abs()
        step = (torch.frexp(y)[1] - 2).clamp(min=-1)  # a half up to 2, one up to 4, two beyond
        y = torch.ldexp(torch.round(torch.ldexp(y, -step)), step)
        code = (y * 2 - (y - 2).clamp(min=0) - (y - 4).clamp(min=0) / 2).to(torch.uint8)
        code = code + 8 * torch.signbit(x).to(torch.uint8)
        return code.view(N, -1)[:, :K].contiguous(), (e[..., 0] + 127).to(torch.uint8), None
    if c["zeros"]:
        lo, hi = x.amin(-1, keepdim=True).clamp(max=0), x.amax(-1, keepdim=True).clamp(min=0)
        reach, steps = hi.double() - lo.double(), 15
    else:
        lo, reach, steps = None, x.abs().amax(-1, keepdim=True).double(), 7
    # the smallest bf16 value s with steps * s >= reach: the one below the quotient, or one of the next two
    low = ((reach / steps).float().view(torch.int32) >> 16).clamp(min=1) - 1
    up = torch.stack([(low + i << 16).view(torch.float32) for i in range(4)])
    scale = torch.where(steps * up.double() >= reach, up, math.inf).amin(0)
    by = torch.where(scale > 0, scale.double(), 1.0)
    zero = torch.round(-lo.double() / by).clamp(max=15) if c["zeros"] else 8
    code = (torch.round(x.double() / by) + zero).clamp(0, 15).to(torch.uint8)
    zero = zero[..., 0].to(torch.uint8) if c["zeros"] else None
    return code.view(N, -1)[:, :K].contiguous(), scale[..., 0].to(torch.bfloat16), zero


def _from_codes(c, codes, scale, zero):
    """The fp32 matrix that codes [N][K], scales and zero points stand for."""
    G, K = c["group"], c["K"]
    if c["type"] == "e2m1":
        v = torch.tensor(CODES + tuple(-x for x in CODES), device="cuda")[codes.int()]
        return v * torch.exp2(scale.float() - 127).repeat_interleave(G, 1)[:, :K]
    z = 8 if zero is None else zero.float().repeat_interleave(G, 1)[:, :K]
    return (codes.float() - z) * scale.float().repeat_interleave(G, 1)[:, :K]


def _linear(s):
    c = s["c"]
    codes = torch.stack([s["codes"] & 15, s["codes"] >> 4], -1).view(c["N"], c["K"])
    y = s["a"].float() @ _from_codes(c, codes, s["scale"], s["zero"]).T
    if s["bias"] is not None:
        y = y + s["bias"]
    if c["out"] == "resid":
        return s["resid"] + y
    if c["out"] == "f32":
        return y
    return (y.clamp(min=0) if c["out"] == "relu" else y).to(torch.bfloat16)


def _row_codes(x, type_):
    """Codes [..., bytes] and scale bytes [..., 2] of fp32 rows [..., 64] as the cache holds them."""
    if type_ == "bf16":
        return x.to(torch.bfloat16).view(torch.uint8), None
    bits, lowest, top, top_exp = BITS[type_]
    b = x.unflatten(-1, (2, BLOCK))
    m, e = torch.frexp(b.abs().amax(-1, keepdim=True))
    e = torch.where(m == 0, -127, e - top_exp + (m > top).to(e.dtype)).clamp(-127, 127)
    y = torch.ldexp(b, -e)
    step = (torch.frexp(y)[1] - 1).clamp(min=lowest) - bits
    y = torch.ldexp(torch.round(torch.ldexp(y.abs(), -step)), step)
    exp = (torch.frexp(y)[1] - 1).clamp(min=lowest)
    field = torch.where(y >= 2.0 ** lowest, exp - lowest + 1, 0)
    mant = torch.ldexp(y, bits - exp).int() - torch.where(field > 0, 1 << bits, 0)
    code = (field.int() << bits) + mant + (torch.signbit(b).int() << (7 if type_ == "e4m3" else 3))
    code = code.flatten(-2).to(torch.uint8)
    return code if type_ == "e4m3" else code[..., 0::2] | (code[..., 1::2] << 4), (e[..., 0] + 127).to(torch.uint8)


def _row_values(codes, scale, type_):
    """fp32 rows of codes and scale bytes."""
    if type_ == "bf16":
        return codes.view(torch.bfloat16).float()
    bits, lowest = BITS[type_][:2]
    n = (codes if type_ == "e4m3" else torch.stack([codes & 15, codes >> 4], -1).flatten(-2)).int()
    mag = n & (127 if type_ == "e4m3" else 7)
    field = mag >> bits
    whole = (mag & ((1 << bits) - 1)) + torch.where(field > 0, 1 << bits, 0)
    y = torch.ldexp(whole.float(), field.clamp(min=1) - 1 + lowest - bits)
    y = torch.where(n > (127 if type_ == "e4m3" else 7), -y, y).unflatten(-1, (2, BLOCK))
    return torch.ldexp(y, scale.int()[..., None] - 127).flatten(-2)


def _places(s):
    """Position, page and place in it of every new token, [T] each."""
    T, page = s["x"].shape[0], s["c"]["page"]
    seq = torch.repeat_interleave(torch.arange(len(s["news"]), device="cuda"), s["first"][1:] - s["first"][:-1],
                                  output_size=T)
    pos = s["len"][seq] - s["first"][seq + 1] + torch.arange(T, device="cuda")
    return pos, s["table"][seq, pos // page].long(), pos % page


def _turn(x, cos, sin, rot, inter):
    """Pairs of the first ``rot`` of the last axis turned by the angles of cos and sin [..., rot / 2]."""
    y = x.clone()
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if inter else (slice(0, rot // 2), slice(rot // 2, rot))
    y[..., first] = x[..., first] * cos - x[..., second] * sin
    y[..., second] = x[..., first] * sin + x[..., second] * cos
    return y


def _append(s):
    c = s["c"]
    H, Hkv, type_ = c["H"], c["Hkv"], c["type"]
    turned = H if c["shared"] else H + Hkv
    pos, page, place = _places(s)
    angle = pos.double()[:, None, None] * s["freq"].double()
    cos, sin = angle.cos().float(), angle.sin().float()
    x = s["x"].float().view(len(pos), -1, D)
    y = x[:, :turned]
    if c["norm"]:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS)
        gain = s["gq"].expand(H, D)
        y = y * (gain if c["shared"] else torch.cat([gain, s["gk"].expand(Hkv, D)]))
    y = _turn(y, cos, sin, c["rot"], c["inter"])
    q, k, v = y[:, :H].to(torch.bfloat16), y[:, turned - Hkv:], x[:, turned:]
    k_codes, k_scale = _row_codes(k, type_)
    v_codes, v_scale = _row_codes(v, type_)
    s["k"][page, :, place], s["v"][page, :, place] = k_codes, v_codes
    if k_scale is not None:
        s["k_scale"][page, :, place], s["v_scale"][page, :, place] = k_scale, v_scale
    if c["shared"]:
        s["k_inv"][page, :, place] = 1 / _row_values(k_codes, k_scale, type_).square().sum(-1).sqrt()
    # the new rows, as the cache holds them
    at = [None if s[n] is None else s[n][page, :, place] for n in ("k", "k_scale", "v", "v_scale")]
    k, v = _row_values(*at[:2], type_), _row_values(*at[2:], type_)
    if c["shared"]:
        k = k * s["k_inv"][page, :, place][..., None]
    return q, k.to(torch.bfloat16), v.to(torch.bfloat16)


def _norm(x, kind):
    """The normalised rows and the factors 1 / deviation."""
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    return x * r, r


def _norm_back(d, n, r, kind):
    """The gradient of a norm's input, from that of its output n."""
    d = d - n * (d * n).mean(-1, keepdim=True)
    return r * (d - d.mean(-1, keepdim=True) if kind == "layer" else d)


def _affine(n, g, b):
    return n * g if b is None else n * g + b


def _residual(s):
    c = s["c"]
    kind = c["norm"]
    f, gate = s["f"].float(), 1.0
    if c["post"]:
        fn, fr = _norm(f, kind)
        u = _affine(fn, s["post_g"], s["post_b"])
    else:
        u = f
    if c["gate"] != "none":
        gate = s["gate"].float()
        gate = 1 / (1 + torch.exp(-gate)) if c["gate"] == "sigmoid" else gate
    scale = 1.0 if s["scale"] is None else s["scale"]
    y = s["x"] + scale * gate * u
    out = {"y": y}
    if c["pre"]:
        yn, yr = _norm(y, kind)
        out["z"] = _affine(yn, s["pre_g"], s["pre_b"]).to(_dtype(c))
    if not c["train"]:
        return out
    dx = s["dy"]
    if c["pre"]:
        out["dpre_g"] = (s["dz"] * yn).sum(0)
        if c["bias"]:
            out["dpre_b"] = s["dz"].sum(0)
        dx = dx + _norm_back(s["dz"] * s["pre_g"], yn, yr, kind)
    out["dx"] = dx
    if c["gate"] != "none":
        slope = gate * (1 - gate) if c["gate"] == "sigmoid" else 1.0
        out["dgate"] = dx * u * scale * slope
    if c["scale"]:
        out["dscale"] = (dx * u * gate).sum(0)
    du = dx * (scale * gate)
    if c["post"]:
        out["dpost_g"] = (du * fn).sum(0)
        if c["bias"]:
            out["dpost_b"] = du.sum(0)
        du = _norm_back(du * s["post_g"], fn, fr, kind)
    out["df"] = du
    return out


# ----------------------------------------------------------------------------
# one pass


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_plain(s):
    c = s["c"]
    if c["kind"] == "linear":
        return _linear(s)
    if c["kind"] == "quantise":
        return _from_codes(c, *_to_codes(c, s["w"]))
    return _append(s) if c["kind"] == "append" else _residual(s)


def _run_own(s):
    c = s["c"]
    if c["kind"] == "linear":
        from paper_2001_04451_amd import w4
        dt = torch.float32 if c["out"] in ("f32", "resid") else torch.bfloat16
        return w4.lsh_linear_w4(s["cfg"], s["a"], s["packed"], bias=s["bias"], resid=s["resid"], relu=c["out"] == "relu",
                                dtype=dt, workspace=s["workspace"])
    if c["kind"] == "quantise":
        from paper_2001_04451_amd import w4
        return w4.lsh_w4_unpack(s["cfg"], w4.lsh_w4_quantize(s["cfg"], s["w"]), torch.float32)
    if c["kind"] == "append":
        from paper_2001_04451_amd import cache
        q = cache.lsh_cache_append(s["cfg"], s["qk"], s["pages"], s["seqs"], s["x"], s["gq"], s["gk"], s["freq"])
        return (q, *cache.lsh_cache_read(s["cfg"], s["pages"], s["seqs"], torch.bfloat16))
    from paper_2001_04451_amd import residual
    y, z = residual.lsh_residual_norm_fwd(s["cfg"], s["x"], s["f"], s["gate"], s["weights"])
    out = {"y": y} if z is None else {"y": y, "z": z}
    if c["train"]:
        grads = residual.lsh_residual_norm_bwd(s["cfg"], y, s["f"], s["gate"], s["weights"], s["dy"], s["dz"])
        out.update({n: t for n, t in grads.items() if t is not None})
    return out


def work(case):
    c = case
    if c["kind"] in ("linear", "quantise"):
        N, K, groups = c["N"], c["K"], -(-c["K"] // c["group"])
        held = N * K // 2 + N * groups * (1 if c["type"] == "e2m1" else 3 if c["zeros"] else 2)
        if c["kind"] == "quantise":
            return {"bytes": N * K * (4 if c["dtype"] == "f32" else 2) + 2 * held + 4 * N * K, "flops": 4 * N * K}
        outs = c["M"] * N * {"relu": 2, "bf16": 2, "f32": 4, "resid": 8}[c["out"]] + (4 * N if c["bias"] else 0)
        return {"bytes": held + 2 * c["M"] * K + outs, "flops": 2 * c["M"] * N * K}
    if c["kind"] == "append":
        T, H, Hkv = sum(_counts(c)[0]), c["H"], c["Hkv"]
        turned = H if c["shared"] else H + Hkv
        held = T * Hkv * (2 * {"bf16": 128, "e4m3": 66, "e2m1": 34}[c["type"]] + (4 if c["shared"] else 0))
        rows = T * (turned + Hkv) * D * (4 if c["dtype"] == "f32" else 2)
        return {"bytes": rows + T * H * D * 2 + 2 * held + T * Hkv * D * 4, "flops": T * (turned * 10 + Hkv * 12) * D}
    n, e = c["T"] * c["D"], 4 if c["dtype"] == "f32" else 2
    gate = c["gate"] != "none"
    bytes_ = n * (4 + e + (e if gate else 0) + 4 + (e if c["pre"] else 0))
    flops = n * 16
    if c["train"]:  # the stream, the branch and the gate are read once more: the backward is another call
        bytes_ += n * (4 + e + (e if gate else 0) + 4 + (4 if c["pre"] else 0) + 4 + 4 + (4 if gate else 0))
        flops += n * 36
    return {"bytes": bytes_, "flops": flops}


# ----------------------------------------------------------------------------
# 64 bits, apart from the above


def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _exact_linear, "quantise": _exact_quantise, "append": _exact_append,
            "residual": _exact_residual}[case["kind"]](s)


def _exact_linear(s):
    c = s["c"]
    packed = s["codes"].long()
    codes = torch.empty(c["N"], c["K"], dtype=torch.long, device="cuda")
    codes[:, 0::2], codes[:, 1::2] = packed % 16, packed // 16
    at = torch.arange(c["K"], device="cuda") // c["group"]
    if c["type"] == "e2m1":
        value = torch.tensor(CODES, dtype=torch.float64, device="cuda")[codes % 8]
        w = torch.where(codes >= 8, -value, value) * 2.0 ** (s["scale"].double() - 127)[:, at]
    else:
        zero = torch.full_like(s["scale"], 8).double() if s["zero"] is None else s["zero"].double()
        w = s["scale"].double()[:, at] * (codes - zero[:, at])
    y = torch.mm(s["a"].double(), w.t())
    y = y if s["bias"] is None else y + s["bias"].double()
    if c["out"] == "relu":
        return torch.relu(y)
    return s["resid"].double() + y if c["out"] == "resid" else y


def _near(x, values):
    """The nearest of the ascending non-negative `values` to |x|, as an index; ties to the even index."""
    mid = (values[1:] + values[:-1]) / 2
    lo, hi = torch.bucketize(x.abs(), mid, right=False), torch.bucketize(x.abs(), mid, right=True)
    return torch.where(lo == hi, lo, torch.where(lo % 2 == 0, lo, hi))


def _power(reach, most):
    """The smallest power of two s with most * s >= reach, 2^-127 at least (and for nothing)."""
    e = torch.floor(torch.log2(torch.where(reach > 0, reach, 1.0) / most)) - 1
    for _ in range(3):
        e = torch.where(most * torch.exp2(e) < reach, e + 1, e)
    return torch.exp2(torch.where(reach > 0, e.clamp(min=-127), -127.0))


def _exact_quantise(s):
    c = s["c"]
    N, K, G = c["N"], c["K"], c["group"]
    out = torch.empty(N, K, dtype=torch.float64, device="cuda")
    every = torch.arange(1 << 15, dtype=torch.int32, device="cuda")[:0x7F80]
    bf16 = (every << 16).view(torch.float32).double()  # every finite one from zero on
    for k0 in range(0, K, G):
        x = s["w"][:, k0:k0 + G].double()
        if c["type"] == "e2m1":
            values = torch.tensor(CODES, dtype=torch.float64, device="cuda")
            by = _power(x.abs().max(1, keepdim=True)[0], 6)
            out[:, k0:k0 + G] = torch.copysign(values[_near(x / by, values)], x) * by
            continue
        lo, hi = x.min(1, keepdim=True)[0], x.max(1, keepdim=True)[0]
        if c["zeros"]:
            lo, hi = torch.minimum(lo, torch.zeros_like(lo)), torch.maximum(hi, torch.zeros_like(hi))
            by = bf16[torch.searchsorted(15 * bf16, hi - lo)]
        else:
            by = bf16[torch.searchsorted(7 * bf16, torch.maximum(-lo, hi))]
        some = torch.where(by > 0, by, torch.ones_like(by))
        zero = torch.round(-lo / some).clamp(max=15) if c["zeros"] else torch.full_like(by, 8)
        out[:, k0:k0 + G] = ((x / some).round().add(zero).clamp(0, 15) - zero) * by
    return out


def _held64(x, type_):
    """fp64 rows as the cache holds them."""
    if type_ == "bf16":
        return x.to(torch.bfloat16).double()
    if type_ == "e2m1":
        values = CODES
    else:
        values = [m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** e for e in range(-9, 6) for m in range(8)][:-1]
    values = torch.tensor(values, dtype=torch.float64, device="cuda")
    halves = torch.stack(x.split(BLOCK, -1), -2)
    by = _power(halves.abs().max(-1, keepdim=True)[0], float(values[-1]))
    y = torch.copysign(values[_near(halves / by, values)], halves) * by
    return torch.cat(y.unbind(-2), -1)


def _exact_append(s):
    c = s["c"]
    H, Hkv, rot = c["H"], c["Hkv"], c["rot"]
    pos = torch.cat([torch.arange(m - n, m, device="cuda") for n, m in zip(*_counts(c))]).double()
    turn = torch.polar(torch.ones(len(pos), rot // 2, dtype=torch.float64, device="cuda"), pos[:, None] * s["freq"].double())
    pair = torch.arange(rot, device="cuda")
    pair = pair.view(-1, 2).T if c["inter"] else pair.view(2, -1)  # the two dimensions of every pair
    x = s["x"].double().view(len(pos), -1, D)

    def heads(a, b, gain):
        y = x[:, a:b]
        if c["norm"]:
            y = y / (y.pow(2).sum(-1, keepdim=True) / D + EPS).sqrt() * gain.double()
        y = y.clone()
        z = torch.complex(y[..., pair[0]], y[..., pair[1]]) * turn[:, None]
        y[..., pair[0]], y[..., pair[1]] = z.real, z.imag
        return y

    q = heads(0, H, s["gq"])
    k = q if c["shared"] else heads(H, H + Hkv, s["gk"])
    k, v = _held64(k, c["type"]), _held64(x[:, -Hkv:], c["type"])
    return q, k / k.norm(dim=-1, keepdim=True) if c["shared"] else k, v


def _exact_residual(s):
    c = s["c"]
    W = c["D"]
    f, x = s["f"].double(), s["x"].double()
    gain = {n: None if s[n] is None else s[n].double() for n in ("scale", "post_g", "post_b", "pre_g", "pre_b")}

    def normed(t, which):
        mean = t.sum(-1, keepdim=True) / W if c["norm"] == "layer" else 0.0
        dev = ((t - mean).pow(2).sum(-1, keepdim=True) / W + EPS).sqrt()
        n = (t - mean) / dev
        y = n * gain[which + "_g"]
        return y if gain[which + "_b"] is None else y + gain[which + "_b"], n, dev

    def through(d, which, n, dev):
        """Gradients of a norm's input, gain and bias."""
        w = d * gain[which + "_g"]
        inner = w - n * (w * n).sum(-1, keepdim=True) / W
        if c["norm"] == "layer":
            inner = inner - w.sum(-1, keepdim=True) / W
        return inner / dev, (d * n).sum(0), d.sum(0)

    u, fn, fdev = normed(f, "post") if c["post"] else (f, None, None)
    raw = torch.ones_like(f) if s["gate"] is None else s["gate"].double()
    gate = torch.sigmoid(raw) if c["gate"] == "sigmoid" else raw
    scale = torch.ones(W, dtype=torch.float64, device="cuda") if gain["scale"] is None else gain["scale"]
    y = x + u * gate * scale
    out = {"y": y}
    if c["pre"]:
        out["z"], yn, ydev = normed(y, "pre")
    if not c["train"]:
        return out
    # the gradients are those at the y that the forward hands over, which is rounded once
    dx = s["dy"].double()
    if c["pre"]:
        _, yn, ydev = normed(y.float().double(), "pre")
        more, out["dpre_g"], db = through(s["dz"].double(), "pre", yn, ydev)
        dx = dx + more
        if c["bias"]:
            out["dpre_b"] = db
    out["dx"] = dx
    if c["gate"] != "none":
        out["dgate"] = dx * u * scale * (gate * torch.sigmoid(-raw) if c["gate"] == "sigmoid" else 1.0)
    if c["scale"]:
        out["dscale"] = (dx * u * gate).sum(0)
    df = dx * gate * scale
    if c["post"]:
        df, out["dpost_g"], db = through(df, "post", fn, fdev)
        if c["bias"]:
            out["dpost_b"] = db
    out["df"] = df
    return out
