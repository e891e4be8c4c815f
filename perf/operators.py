"""The work the cache, its attention and the per-head norm are measured on.

``listed()`` names the cases, ``draw()`` gives others of the same ranges, ``prepare`` makes what a program
holds before the call, ``run`` is one pass (elementary torch in 32 bits, or with ``own`` the library's
calls), ``work`` the bytes and operations a pass cannot do without, ``exact`` the outputs in 64 bits.

Kinds of case:
  rotate  per-head norm and position rotation of projected rows; with ``train`` the backward too;
  write   new tokens' rows quantised into the paged cache, and those rows read back;
  read    whole sequences read back from the cache, as rows for a pass over the full context;
  attn    new tokens attending to their sequences' cached rows (one token each: decoding).
"""
import math
import random

import torch

own = False

D = 64  # head width
BLOCK = 32  # values that share a scale
LARGEST = {"e4m3": 448.0, "e2m1": 6.0}  # largest value of a code
LOWEST_EXP = {"e4m3": -6, "e2m1": 0}  # exponent of the smallest normal value
MANTISSA = {"e4m3": 3, "e2m1": 1}
ROW_BYTES = {"bf16": 128, "e4m3": 66, "e2m1": 34}  # codes and scales of a row
EPS = 1e-6
SELF_MASK = 1e5


def listed():
    return [
        # one decoding step's queries: 64 sequences, 16 heads, positions anywhere in 64K
        dict(name="rotate_decode_64", kind="rotate", dtype="bf16", B=64, L=1, Hq=16, Hk=0, rot=64, inter=False,
             per_head=False, train=False, pos0=40000, heads_first=False),
        # fp32 fine-tuning on a ragged batch, separate keys on fewer heads, half the width rotated; both directions
        dict(name="rotate_f32_ragged_train", kind="rotate", dtype="f32", B=3, L=1999, Hq=8, Hk=2, rot=32, inter=True,
             per_head=True, train=True, pos0=0, heads_first=True),
        # the training batch of the LSH attention: 8 sequences of 32K, 8 heads, both directions
        dict(name="rotate_bf16_32k_train", kind="rotate", dtype="bf16", B=8, L=32768, Hq=8, Hk=0, rot=64, inter=False,
             per_head=False, train=True, pos0=0, heads_first=True),
        # a decoding step's rows into an e4m3 cache: 64 sequences, 16 heads
        dict(name="write_decode_64", kind="write", dtype="bf16", type="e4m3", n_seq=64, new=1, new_rest=1, H=16, Hkv=16,
             len=8000, ragged=True, page=64, shared=True),
        # a long prompt into a 4-bit cache, fp32 rows
        dict(name="write_prompt_e2m1", kind="write", dtype="f32", type="e2m1", n_seq=1, new=16384, new_rest=1, H=16,
             Hkv=16, len=16384, ragged=False, page=64, shared=True),
        # several contexts read back from the cache, for an LSH pass over all of them
        dict(name="read_e4m3_8x8k", kind="read", dtype="bf16", type="e4m3", n_seq=8, H=16, Hkv=16, len=8191, ragged=True,
             page=16, shared=True),
        # the smallest call: one sequence's next token
        dict(name="attn_one_1k", kind="attn", type="bf16", n_seq=1, new=1, new_rest=1, H=8, Hkv=8, len=1000,
             ragged=False, page=16, shared=True),
        # a serving batch's decoding step, lengths from hundreds to 16K
        dict(name="attn_decode_64_ragged", kind="attn", type="e4m3", n_seq=64, new=1, new_rest=1, H=16, Hkv=16,
             len=16384, ragged=True, page=64, shared=True),
        # grouped heads over a 4-bit cache, 32 contexts of 32K
        dict(name="attn_decode_grouped_32k", kind="attn", type="e2m1", n_seq=32, new=1, new_rest=1, H=16, Hkv=2,
             len=32768, ragged=False, page=128, shared=False),
        # the paper's longest context, one sequence, 16 heads: nothing but the length to split
        dict(name="attn_decode_64k", kind="attn", type="bf16", n_seq=1, new=1, new_rest=1, H=16, Hkv=16, len=65536,
             ragged=False, page=64, shared=True),
        # a step that mixes a chunk of a prompt with decoding sequences
        dict(name="attn_mixed_grouped", kind="attn", type="bf16", n_seq=32, new=512, new_rest=1, H=16, Hkv=4, len=6001,
             ragged=True, page=32, shared=False),
        # a chunk of a long prompt over what is cached of it
        dict(name="attn_chunk_2k_32k", kind="attn", type="e4m3", n_seq=1, new=2048, new_rest=1, H=16, Hkv=16, len=32768,
             ragged=False, page=64, shared=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "rotate", "write", "read", "attn", "attn", "attn", "attn"])
    if kind == "rotate":
        Hq = rng.choice([1, 2, 4, 8, 12, 16])
        Hk = rng.choice([0, 0] + [h for h in (1, 2, 4, Hq) if Hq % h == 0])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        L = _log(rng, 1, 32768)
        B = _log(rng, 1, max(1, min(64, (262144 * 8 // (2 if dtype == "f32" else 1)) // (L * (Hq + Hk)))))
        return dict(kind=kind, dtype=dtype, B=B, L=L, Hq=Hq, Hk=Hk, rot=rng.choice([64, 64, 32, 16, 48]),
                    inter=rng.random() < 0.5, per_head=rng.random() < 0.5, train=rng.random() < 0.6,
                    pos0=rng.choice([0, 0, _log(rng, 1, 1 << 24)]), heads_first=rng.random() < 0.6)
    type_ = rng.choice(["bf16", "e4m3", "e4m3", "e2m1"])
    page = rng.choice([16, 32, 64, 64, 128, 256])
    shared = rng.random() < 0.6
    H = rng.choice([1, 2, 4, 8, 8, 16, 16])
    Hkv = H if shared else rng.choice([h for h in (1, 2, 4, 8, 16) if H % h == 0])
    if kind == "write":
        new = _log(rng, 1, 16384)
        n_seq = _log(rng, 1, max(1, min(128, 16384 // new)))
        return dict(kind=kind, dtype=rng.choice(["bf16", "f32"]), type=type_, n_seq=n_seq, new=new, new_rest=new, H=H,
                    Hkv=Hkv, len=new + _log(rng, 1, max(1, min(8192, (1 << 18) // n_seq))), ragged=rng.random() < 0.5,
                    page=page, shared=shared)
    if kind == "read":
        length = _log(rng, 1, 32768)
        n_seq = _log(rng, 1, max(1, min(128, 32768 // length)))
        return dict(kind=kind, dtype=rng.choice(["bf16", "f32"]), type=type_, n_seq=n_seq, H=H, Hkv=Hkv, len=length,
                    ragged=rng.random() < 0.5, page=page, shared=shared)
    length = _log(rng, 1, 65536)
    how = rng.randrange(4)
    if how < 2:  # decoding
        new = new_rest = 1
        n_seq = _log(rng, 1, max(1, min(128, (1 << 22) // (length * Hkv))))
    elif how == 2:  # a few tokens each
        new = new_rest = min(length, rng.randint(2, 24))
        n_seq = _log(rng, 1, max(1, min(64, (1 << 18) // length)))
    else:  # a chunk, alone or beside decoding sequences
        new, new_rest = min(length, _log(rng, 16, 2048), (3 << 24) // length), 1
        n_seq = rng.choice([1, 1, _log(rng, 1, max(1, min(32, (1 << 18) // length)))])
    return dict(kind="attn", type=type_, n_seq=n_seq, new=new, new_rest=new_rest, H=H, Hkv=Hkv, len=length,
                ragged=rng.random() < 0.5, page=page, shared=shared)


def _counts(c):
    """New (or read) tokens and cached length of each sequence; from the case alone."""
    n = c["n_seq"]
    if c["ragged"]:  # spread over the length's logarithm, down to a thirty-second, in a fixed disorder
        lens = [max(1, int(round(c["len"] * 32.0 ** (-i / max(1, n - 1))))) for i in range(n)]
        random.Random(n * 1000003 + c["len"]).shuffle(lens)
    else:
        lens = [c["len"]] * n
    if c["kind"] == "read":
        return lens, lens
    news = [c["new"]] + [c["new_rest"]] * (n - 1)
    return news, [max(a, b) for a, b in zip(lens, news)]


# ----------------------------------------------------------------------------
# inputs


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return _prepare_rotate(case, g) if case["kind"] == "rotate" else _prepare_cache(case, g)


def _prepare_rotate(c, g):
    B, L, Hq, Hk, rot = c["B"], c["L"], c["Hq"], c["Hk"], c["rot"]
    T, dt = B * L, _dtype(c)
    # channels of unequal size, as a projection gives them
    size = torch.exp(0.5 * _randn(g, (Hq + Hk) * D))
    s = {"c": c, "x": (_randn(g, T, (Hq + Hk) * D) * size).to(dt)}
    s["gq"] = 1 + 0.1 * _randn(g, *((Hq, D) if c["per_head"] else (D,)))
    s["gk"] = 1 + 0.1 * _randn(g, *((Hk, D) if c["per_head"] else (D,))) if Hk else None
    s["freq"] = (10000.0 ** (-torch.arange(rot // 2, device="cuda", dtype=torch.float64) * 2 / rot)).float()
    if L == 1:  # decoding: every sequence at its own position
        pos = c["pos0"] + torch.randint(0, 20000, (B,), generator=g, device="cuda")
    else:
        pos = c["pos0"] + torch.arange(L, device="cuda").repeat(B)
    s["pos"] = pos.to(torch.int32)
    if c["train"]:
        s["dq"] = _randn(g, *_out_shape(c, Hq))
        s["dk"] = _randn(g, *_out_shape(c, Hk)) if Hk else None
    if own:
        from paper_2001_04451_amd import qk
        s["cfg"] = qk.QkConfig(T=T, Hq=Hq, Hk=Hk, rot=rot, interleaved=c["inter"], gain_per_head=c["per_head"], eps=EPS,
                               L=L if c["heads_first"] else 0)
    return s


def _out_shape(c, H):
    return (c["B"], H, c["L"], D) if c["heads_first"] else (c["B"] * c["L"], H, D)


def _prepare_cache(c, g):
    news, lens = _counts(c)
    H, Hkv, page, type_ = c["H"], c["Hkv"], c["page"], c["type"]
    n_seq, T = c["n_seq"], sum(news)
    used = [-(-n // page) for n in lens]
    n_pages, most = sum(used) + 3, max(used)
    where = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((n_seq, most), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(used):
        table[i, :n] = where[at:at + n]
        at += n
    first = torch.tensor([sum(news[:i]) for i in range(n_seq + 1)], dtype=torch.int32, device="cuda")
    s = {"c": c, "first": first, "len": torch.tensor(lens, dtype=torch.int32, device="cuda"), "table": table,
         "news": news, "lens": lens}
    s.update(_fill_pages(c, g, n_pages))
    if c["kind"] == "write":
        s["k"] = _rows(g, T, Hkv).to(_dtype(c))
        s["v"] = _randn(g, T, Hkv, D).to(_dtype(c))
    if c["kind"] == "attn":
        s["q"] = _rows(g, T, H).to(torch.bfloat16)
    if own:
        from paper_2001_04451_amd import cache
        s["cfg"] = cache.CacheConfig(n_seq=n_seq, T=T, H=H, Hkv=Hkv, n_pages=n_pages, max_pages=most, page=page,
                                     type=type_, shared_qk=c["shared"], self_mask=SELF_MASK, max_new=max(news))
        s["pages"] = cache.Pages(k=s["k_codes"], v=s["v_codes"], k_scale=s["k_scale"], v_scale=s["v_scale"],
                                 k_inv=s["k_inv"])
        s["seqs"] = cache.Sequences(first=s["first"], length=s["len"], table=s["table"])
        if c["kind"] == "attn":
            s["out"] = torch.empty(T, H, D, dtype=torch.bfloat16, device="cuda")
            s["lse"] = torch.empty(T, H, dtype=torch.float32, device="cuda")
            s["workspace"] = cache.workspace(s["cfg"], s["out"].device)
    return s


def _rows(g, n, H):
    """Query or key rows: Gaussians of unequal length, as projections give them."""
    return _randn(g, n, H, D) * torch.exp(0.3 * _randn(g, n, H, 1))


def _fill_pages(c, g, n_pages):
    """A pool of pages whose every slot holds a row (slots past a sequence's end: some earlier one's)."""
    Hkv, page, type_ = c["Hkv"], c["page"], c["type"]
    n = n_pages * Hkv * page
    bytes_ = {"bf16": 2 * D, "e4m3": D, "e2m1": D // 2}[type_]
    out = {"k_scale": None, "v_scale": None, "k_inv": None}
    for x in "kv":
        codes = torch.empty(n, bytes_, dtype=torch.uint8, device="cuda")
        scale = None if type_ == "bf16" else torch.empty(n, 2, dtype=torch.uint8, device="cuda")
        inv = torch.empty(n, dtype=torch.float32, device="cuda")
        for a in range(0, n, 1 << 20):
            b = min(n, a + (1 << 20))
            r = _rows(g, b - a, 1)[:, 0] if x == "k" else _randn(g, b - a, D)
            cd, sc = _quantise(r.to(torch.bfloat16).float(), type_)
            codes[a:b] = cd
            if sc is not None:
                scale[a:b] = sc
            if x == "k" and c["shared"]:
                inv[a:b] = 1 / _values(cd, sc, type_).double().square().sum(-1).sqrt()
        out[x + "_codes"] = codes.view(n_pages, Hkv, page, bytes_)
        if scale is not None:
            out[x + "_scale"] = scale.view(n_pages, Hkv, page, 2)
        if x == "k" and c["shared"]:
            out["k_inv"] = inv.view(n_pages, Hkv, page)
    return out


# ----------------------------------------------------------------------------
# the plain forms


def _quantise(x, type_):
    """Codes [..., bytes] and scale bytes [..., 2] of fp32 rows [..., 64]; every step but one rounding is exact."""
    if type_ == "bf16":
        return x.to(torch.bfloat16).view(torch.uint8), None
    b = x.reshape(*x.shape[:-1], 2, BLOCK)
    m, e = torch.frexp(b.abs().amax(-1, keepdim=True))  # amax = m 2^e, m in [0.5, 1)
    # the smallest exponent that brings the block's largest magnitude to LARGEST or below
    top = {"e4m3": (0.875, 9), "e2m1": (0.75, 3)}[type_]  # LARGEST = 0.875 * 2^9, 0.75 * 2^3
    e = e - top[1] + (m > top[0]).to(e.dtype)
    e = torch.where(m == 0, torch.full_like(e, -127), e).clamp(-127, 127)
    y = torch.ldexp(b, -e)
    _, ey = torch.frexp(y)
    step = (ey - 1).clamp(min=LOWEST_EXP[type_]) - MANTISSA[type_]
    n = torch.round(torch.ldexp(y.abs(), -step))  # half to even
    a = torch.ldexp(n, step)  # the value the code stands for, unscaled
    # code: exponent field and mantissa of a
    _, ea = torch.frexp(a)
    field = torch.where(a >= 2.0 ** LOWEST_EXP[type_], ea - 1 - LOWEST_EXP[type_] + 1, torch.zeros_like(ea))
    st = (ea - 1).clamp(min=LOWEST_EXP[type_]) - MANTISSA[type_]
    mant = torch.ldexp(a, -st).to(torch.int32) - torch.where(field > 0, 1 << MANTISSA[type_], 0)
    sign = torch.signbit(b).to(torch.int32)
    code = (sign << (7 if type_ == "e4m3" else 3)) | (field.to(torch.int32) << MANTISSA[type_]) | mant
    code = code.reshape(x.shape).to(torch.uint8)
    if type_ == "e2m1":  # two values a byte, the even one in the low half
        code = code[..., 0::2] | (code[..., 1::2] << 4)
    return code, (e[..., 0] + 127).to(torch.uint8)


def _values(codes, scale, type_):
    """fp32 rows of codes and scale bytes."""
    if type_ == "bf16":
        return codes.view(torch.bfloat16).float()
    if type_ == "e4m3":
        n = codes.to(torch.int32)
        sign, field, mant = n >> 7, (n >> 3) & 15, n & 7
    else:
        n = torch.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], D).to(torch.int32)
        sign, field, mant = n >> 3, (n >> 1) & 3, n & 1
    whole = torch.where(field > 0, mant + (1 << MANTISSA[type_]), mant).float()
    a = torch.ldexp(whole, field.clamp(min=1) - 1 + LOWEST_EXP[type_] - MANTISSA[type_])
    a = torch.where(sign > 0, -a, a).reshape(*codes.shape[:-1], 2, BLOCK)
    return torch.ldexp(a, scale.to(torch.int32)[..., None] - 127).reshape(*codes.shape[:-1], D)


def _slots(s):
    """Page and place in it of every new (or read) token, [T] each."""
    page, table = s["c"]["page"], s["table"]
    seq = torch.repeat_interleave(torch.arange(len(s["news"]), device="cuda"), s["first"][1:] - s["first"][:-1],
                                  output_size=sum(s["news"]))
    t = torch.arange(sum(s["news"]), device="cuda")
    pos = s["len"][seq] - (s["first"][seq + 1] - t)
    return table[seq, pos // page].long(), pos % page


def _read(s):
    """Rows of the new (or read) tokens as the cache holds them, [T][Hkv][64] in the case's type."""
    c = s["c"]
    p, o = _slots(s)
    rows = []
    for x in "kv":
        sc = s[x + "_scale"]
        r = _values(s[x + "_codes"][p, :, o], None if sc is None else sc[p, :, o], c["type"])
        if x == "k" and c["shared"]:
            r = r * s["k_inv"][p, :, o][..., None]
        rows.append(r.to(_dtype(c)))
    return tuple(rows)


def _write(s):
    c = s["c"]
    p, o = _slots(s)
    for x in "kv":
        codes, scale = _quantise(s[x].float(), c["type"])
        s[x + "_codes"][p, :, o] = codes
        if scale is not None:
            s[x + "_scale"][p, :, o] = scale
        if x == "k" and c["shared"]:
            r = _values(codes, scale, c["type"])
            s["k_inv"][p, :, o] = 1 / r.square().sum(-1).sqrt()


def _attend(s):
    c = s["c"]
    H, Hkv, page = c["H"], c["Hkv"], c["page"]
    G = H // Hkv
    outs, lses = [], []
    t = 0
    for i, (n, length) in enumerate(zip(s["news"], s["lens"])):
        ids = s["table"][i, : -(-length // page)].long()

        def rows(x):
            sc = s[x + "_scale"]
            r = _values(s[x + "_codes"][ids], None if sc is None else sc[ids], c["type"])  # [pages][Hkv][page][64]
            if x == "k" and c["shared"]:
                r = r * s["k_inv"][ids][..., None]
            return r.transpose(0, 1).reshape(Hkv, -1, D)[:, :length]

        k, v = rows("k"), rows("v")
        q = s["q"][t:t + n].float().reshape(n, Hkv, G, D).permute(1, 2, 0, 3).reshape(Hkv, G * n, D)
        z = torch.bmm(q, k.transpose(1, 2).contiguous()).view(Hkv, G, n, length) / math.sqrt(D)
        pos = length - n + torch.arange(n, device="cuda")
        key = torch.arange(length, device="cuda")
        if c["shared"]:
            z = z - SELF_MASK * (key[None, :] == pos[:, None])
        z = z.masked_fill(key[None, :] > pos[:, None], -math.inf)
        m = z.amax(-1, keepdim=True)
        w = torch.exp(z - m)
        del z
        total = w.sum(-1, keepdim=True)
        o = torch.bmm(w.view(Hkv, G * n, length), v).view(Hkv, G, n, D) / total
        outs.append(o.permute(2, 0, 1, 3).reshape(n, H, D))
        lses.append((m + torch.log(total))[..., 0].permute(2, 0, 1).reshape(n, H))
        t += n
    return torch.cat(outs).to(torch.bfloat16), torch.cat(lses)


def _turn(x, cos, sin, rot, inter):
    """Pairs of the first ``rot`` of the last axis turned by the angles of cos and sin [..., rot / 2]."""
    y = x.clone()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if inter else (x[..., :rot // 2], x[..., rot // 2:rot])
    ya, yb = a * cos - b * sin, a * sin + b * cos
    if inter:
        y[..., 0:rot:2], y[..., 1:rot:2] = ya, yb
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = ya, yb
    return y


def _rotate(s):
    c = s["c"]
    B, L, Hq, Hk = c["B"], c["L"], c["Hq"], c["Hk"]
    T = B * L
    angle = s["pos"].double()[:, None] * s["freq"].double()
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]  # [T][1][rot / 2]
    x = s["x"].float().view(T, Hq + Hk, D)
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    n = x * r
    outs, grads, gains = [], [], []
    for h0, h1, gain, d in ((0, Hq, s["gq"], s.get("dq")), (Hq, Hq + Hk, s["gk"], s.get("dk"))):
        if h0 == h1:
            continue
        y = _turn(n[:, h0:h1] * gain, cos, sin, c["rot"], c["inter"]).to(_dtype(c))
        if c["heads_first"]:
            y = y.view(B, L, h1 - h0, D).transpose(1, 2).contiguous()
        outs.append(y)
        if c["train"]:
            d = d.transpose(1, 2).reshape(T, h1 - h0, D) if c["heads_first"] else d
            u = _turn(d, cos, -sin, c["rot"], c["inter"])
            nn = n[:, h0:h1]
            gains.append((u * nn).sum(0) if c["per_head"] else (u * nn).sum((0, 1)))
            w = u * gain
            grads.append(r[:, h0:h1] * (w - nn * (w * nn).mean(-1, keepdim=True)))
    if not c["train"]:
        return tuple(outs)
    return (*outs, torch.cat(grads, 1).view(T, -1), *gains)


# ----------------------------------------------------------------------------
# one pass


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_plain(s):
    kind = s["c"]["kind"]
    if kind == "rotate":
        return _rotate(s)
    if kind == "attn":
        return _attend(s)
    if kind == "write":
        _write(s)
    return _read(s)


def _run_own(s):
    c = s["c"]
    if c["kind"] == "rotate":
        from paper_2001_04451_amd import qk
        q, k = qk.lsh_qk_norm_rotate_fwd(s["cfg"], s["x"], s["gq"], s["gk"], s["freq"], s["pos"])
        outs = (q,) if k is None else (q, k)
        if not c["train"]:
            return outs
        dx, dgq, dgk = qk.lsh_qk_norm_rotate_bwd(s["cfg"], s["x"], s["gq"], s["gk"], s["freq"], s["pos"], s["dq"],
                                                 s["dk"])
        return (*outs, dx, dgq) if k is None else (*outs, dx, dgq, dgk)
    from paper_2001_04451_amd import cache
    if c["kind"] == "attn":
        return cache.lsh_cache_attn_fwd(s["cfg"], s["pages"], s["seqs"], s["q"], out=s["out"], lse=s["lse"],
                                        workspace=s["workspace"])
    if c["kind"] == "write":
        cache.lsh_cache_write(s["cfg"], s["pages"], s["seqs"], s["k"], s["v"])
    return cache.lsh_cache_read(s["cfg"], s["pages"], s["seqs"], _dtype(c))


def work(case):
    c = case
    if c["kind"] == "rotate":
        n = c["B"] * c["L"] * (c["Hq"] + c["Hk"]) * D
        e = 4 if c["dtype"] == "f32" else 2
        bytes_, flops = n * 2 * e + c["B"] * c["L"] * 4, n * 7
        if c["train"]:  # x is read once more: the backward is another call
            bytes_, flops = bytes_ + n * (e + 8), flops + n * 12
        return {"bytes": bytes_, "flops": flops}
    news, lens = _counts(c)
    row = ROW_BYTES[c["type"]]
    key = 4 if c["shared"] else 0
    if c["kind"] == "attn":
        # rows that some new token sees; a shared-QK token sees its own only if there is no other
        seen = sum(max(1, n - 1) if c["shared"] else n for n in lens)
        pairs = sum(n * length - n * (n - 1) // 2 - (n if c["shared"] else 0) for n, length in zip(news, lens))
        rows = sum(news) * c["H"]
        return {"bytes": seen * c["Hkv"] * (2 * row + key) + rows * (4 * D + 4), "flops": pairs * c["H"] * 4 * D}
    rows = sum(news) * c["Hkv"]
    e = 4 if c["dtype"] == "f32" else 2
    read = rows * (2 * row + key + 2 * e * D)
    if c["kind"] == "read":
        return {"bytes": read, "flops": rows * 2 * D}
    return {"bytes": 2 * read, "flops": rows * 2 * D * 6}


# ----------------------------------------------------------------------------
# 64 bits, apart from the above


def _table(type_):
    """Every code's value."""
    bits, lowest, man = (8, -6, 3) if type_ == "e4m3" else (4, 0, 1)
    vals = []
    for code in range(1 << bits):
        mag = code & ((1 << (bits - 1)) - 1)
        field, frac = mag >> man, mag & ((1 << man) - 1)
        v = (frac / (1 << man)) * 2.0 ** lowest if field == 0 else (1 + frac / (1 << man)) * 2.0 ** (field - 1 + lowest)
        if type_ == "e4m3" and mag == 127:
            v = math.nan
        vals.append(-v if code >> (bits - 1) else v)
    return torch.tensor(vals, dtype=torch.float64, device="cuda")


def _decode64(codes, scale, type_):
    if type_ == "bf16":
        return codes.view(torch.bfloat16).double()
    idx = codes.long() if type_ == "e4m3" else torch.stack([codes.long() % 16, codes.long() // 16], -1).flatten(-2)
    v = _table(type_)[idx]
    return v * torch.exp2(scale.double() - 127).repeat_interleave(BLOCK, -1)


def _nearest64(x, type_):
    """fp64 rows rounded to the values that codes stand for: the nearest of the table, ties to the even code."""
    if type_ == "bf16":
        return x.to(torch.bfloat16).double()
    top = LARGEST[type_]
    vals = _table(type_)[: 128 if type_ == "e4m3" else 8]
    vals = vals[~vals.isnan()].contiguous()
    mid = ((vals[1:] + vals[:-1]) / 2).contiguous()
    b = x.unflatten(-1, (2, BLOCK))
    amax = b.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(torch.where(amax > 0, amax, torch.ones_like(amax)) / top))
    e = torch.where(amax > top * torch.exp2(e), e + 1, e)  # against log2's rounding
    e = torch.where(amax <= top * torch.exp2(e - 1), e - 1, e)
    e = torch.where(amax > 0, e.clamp(-127, 127), torch.full_like(e, -127))
    y = (b / torch.exp2(e)).abs()
    lo = torch.bucketize(y, mid, right=False)  # codes whose upper midpoint is at or above y
    tie = torch.where(lo < len(mid), mid[lo.clamp(max=len(mid) - 1)] == y, torch.zeros_like(y, dtype=torch.bool))
    code = torch.where(tie & (lo % 2 == 1), lo + 1, lo)
    return (torch.copysign(vals[code], b) * torch.exp2(e)).flatten(-2)


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["kind"] == "rotate":
        return _exact_rotate(s)
    if c["kind"] == "attn":
        return _exact_attend(s)
    if c["kind"] == "write":
        k, v = _nearest64(s["k"].double(), c["type"]), _nearest64(s["v"].double(), c["type"])
        if c["shared"]:
            k = k / k.norm(dim=-1, keepdim=True)
        return k, v
    outs = []
    for x in "kv":
        parts = []
        for i, n in enumerate(s["lens"]):
            ids = s["table"][i, : -(-n // c["page"])].long()
            sc = s[x + "_scale"]
            r = _decode64(s[x + "_codes"][ids], None if sc is None else sc[ids], c["type"])
            parts.append(r.transpose(1, 2).flatten(0, 1)[:n])
        r = torch.cat(parts)
        outs.append(r / r.norm(dim=-1, keepdim=True) if x == "k" and c["shared"] else r)
    return tuple(outs)


def _exact_attend(s):
    c = s["c"]
    H, Hkv = c["H"], c["Hkv"]
    T = sum(s["news"])
    out = torch.empty(T, H, D, dtype=torch.float64, device="cuda")
    lse = torch.empty(T, H, dtype=torch.float64, device="cuda")
    t = 0
    for i, (n, length) in enumerate(zip(s["news"], s["lens"])):
        ids = s["table"][i, : -(-length // c["page"])].long()
        for hk in range(Hkv):
            sk, sv = s["k_scale"], s["v_scale"]
            k = _decode64(s["k_codes"][ids, hk], None if sk is None else sk[ids, hk], c["type"]).flatten(0, 1)[:length]
            v = _decode64(s["v_codes"][ids, hk], None if sv is None else sv[ids, hk], c["type"]).flatten(0, 1)[:length]
            if c["shared"]:
                k = k / k.norm(dim=-1, keepdim=True)
            for h in range(hk * (H // Hkv), (hk + 1) * (H // Hkv)):
                z = s["q"][t:t + n, h].double() @ k.T * D ** -0.5
                ahead = torch.ones(n, length, dtype=torch.bool, device="cuda").tril(length - n)
                if c["shared"]:
                    z.diagonal(length - n).sub_(SELF_MASK)
                z = torch.where(ahead, z, torch.full_like(z, -math.inf))
                lse[t:t + n, h] = torch.logsumexp(z, -1)
                out[t:t + n, h] = torch.softmax(z, -1) @ v
        t += n
    return out, lse


def _exact_rotate(s):
    c = s["c"]
    B, L, Hq, Hk, rot = c["B"], c["L"], c["Hq"], c["Hk"], c["rot"]
    T = B * L
    turn = torch.polar(torch.ones(T, rot // 2, dtype=torch.float64, device="cuda"),
                       s["pos"].double()[:, None] * s["freq"].double())[:, None]
    pair = torch.arange(rot, device="cuda")
    pair = pair.view(-1, 2).T if c["inter"] else pair.view(2, -1)  # the two dims of every pair

    def apply(y, z):
        y = y.clone()
        w = torch.complex(y[..., pair[0]], y[..., pair[1]]) * z
        y[..., pair[0]], y[..., pair[1]] = w.real, w.imag
        return y

    outs, dxs, dgs = [], [], []
    x = s["x"].double().view(T, Hq + Hk, D)
    for hs, gain, d in ((slice(0, Hq), s["gq"], s.get("dq")), (slice(Hq, Hq + Hk), s["gk"], s.get("dk"))):
        if gain is None:
            continue
        xs, gain = x[:, hs], gain.double()
        H = xs.shape[1]
        rms = (xs.pow(2).sum(-1, keepdim=True) / D + EPS).sqrt()
        y = apply(xs / rms * gain, turn)
        outs.append(y.view(B, L, H, D).permute(0, 2, 1, 3).contiguous() if c["heads_first"] else y)
        if c["train"]:
            d = d.double()
            d = d.permute(0, 2, 1, 3).reshape(T, H, D) if c["heads_first"] else d
            u = apply(d, turn.conj())
            dgs.append((u * xs / rms).sum(0) if c["per_head"] else (u * xs / rms).flatten(0, 1).sum(0))
            w = u * gain
            dxs.append(w / rms - xs * (w * xs).sum(-1, keepdim=True) / (D * rms ** 3))
    if not c["train"]:
        return tuple(outs)
    return (*outs, torch.cat(dxs, 1).reshape(T, -1), *dgs)
