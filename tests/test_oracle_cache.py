"""The oracles of the cache and of the per-head norm with rotation, each against an independent form (CPU)."""
import numpy as np
import pytest
import torch

import oracle
from oracle import cache as C
from oracle import qk as Q


def test_code_values():
    assert C.code_values("e2m1").tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    theirs = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(C.code_values("e4m3")[:127], theirs)


def test_encode_e4m3_is_the_scaled_cast():
    x = np.random.default_rng(0).standard_normal((200, 64)).astype(np.float32) * 10.0 ** np.linspace(-6, 6, 200)[:, None]
    x = x.astype(np.float32)
    codes, scale = C.encode(x, "e4m3")
    y = x.reshape(200, 2, 32) * np.exp2(127.0 - scale[..., None])
    assert np.abs(y).max() <= 448 and (np.abs(y).max(-1) > 224).all()
    theirs = torch.from_numpy(y.astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(codes.reshape(200, 2, 32), theirs)


@pytest.mark.parametrize("type_", ["e4m3", "e2m1"])
def test_encode_nearest_and_ties(type_):
    """Values on, half way between and beside the codes' values, in a block whose largest value fixes the scale to one."""
    v = C.code_values(type_)
    v = v[:127] if type_ == "e4m3" else v
    mid = (v[1:] + v[:-1]) / 2
    x = np.concatenate([v, mid, np.nextafter(mid, 0), np.nextafter(mid, 1e9)])
    want = np.concatenate([np.arange(len(v)), np.arange(1, len(v)) // 2 * 2, np.arange(len(mid)), np.arange(1, len(v))])
    for i in range(0, len(x), 31):
        row = np.zeros(64)
        part = x[i:i + 31]
        row[:len(part)], row[31] = -part, v[-1]
        codes, scale = C.encode(row, type_)
        assert scale[0] == 127
        if type_ == "e2m1":
            codes = np.stack([codes & 15, codes >> 4], -1).reshape(-1)
        sign = 128 if type_ == "e4m3" else 8
        assert np.array_equal(codes[:len(part)] & (sign - 1), want[i:i + 31])
        assert np.array_equal(C.decode(*C.encode(row, type_), type_)[:len(part)], -v[want[i:i + 31]])


def test_encode_bf16_and_special_blocks():
    x = np.random.default_rng(1).standard_normal((50, 64)).astype(np.float32)
    assert np.array_equal(C.decode(*C.encode(x, "bf16"), "bf16"),
                          torch.from_numpy(x).to(torch.bfloat16).double().numpy())
    for type_ in ("e4m3", "e2m1"):
        row = np.zeros(64)
        row[40] = np.inf
        codes, scale = C.encode(row, type_)
        assert scale.tolist() == [0, 255] and not codes.any()
        got = C.decode(codes, scale, type_)
        assert (got[:32] == 0).all() and np.isnan(got[32:]).all()


def test_attend_is_the_dense_shared_attention():
    """Whole sequences as new tokens: the dense oracle's causal shared-QK attention."""
    rng = np.random.default_rng(2)
    L, H, page = 37, 2, 16
    q, v = rng.standard_normal((2, H, L, 64))
    table = np.array([[3, 0, 2]], np.int32)
    k_rows, v_rows = np.full((4, H, page, 64), np.nan), np.full((4, H, page, 64), np.nan)
    for j in range(L):
        p = table[0, j // page]
        k_rows[p, :, j % page], v_rows[p, :, j % page] = q[:, j], v[:, j]
    out, lse, _, _ = C.attend(q.transpose(1, 0, 2), k_rows, v_rows, C.inverse_length(k_rows), [0, L], [L], table, page,
                              0.125, True, 1e5)
    ref_out, ref_lse = oracle.dense_attn_fwd(q[None], v[None], True)
    assert np.abs(out.transpose(1, 0, 2) - ref_out[0]).max() < 1e-12
    assert np.abs(lse.T - ref_lse[0]).max() < 1e-9


def test_attend_grouped_and_holes():
    """Grouped heads against torch's softmax in fp64; pages outside the pool are no one's keys."""
    rng = np.random.default_rng(3)
    n, page, H, Hkv = 40, 16, 4, 2
    k_rows, v_rows = rng.standard_normal((2, 3, Hkv, page, 64))
    table = np.array([[1, -1, 0]], np.int32)
    q = rng.standard_normal((3, H, 64))
    out, lse, _, _ = C.attend(q, k_rows, v_rows, None, [0, 3], [n], table, page, 0.2, False, 1e5)
    pos = np.r_[0:16, 32:40]
    K = np.concatenate([k_rows[1], k_rows[0][:, :8]], 1)  # [Hkv][24][64]
    V = np.concatenate([v_rows[1], v_rows[0][:, :8]], 1)
    for i in range(3):
        for h in range(H):
            z = torch.from_numpy(K[h // 2] @ q[i, h] * 0.2)
            z = torch.where(torch.from_numpy(pos <= n - 3 + i), z, -torch.inf)
            assert np.abs((torch.softmax(z, 0) @ torch.from_numpy(V[h // 2])).numpy() - out[i, h]).max() < 1e-12
            assert abs(torch.logsumexp(z, 0).item() - lse[i, h]) < 1e-12
    # nothing at all to see
    out, lse, _, _ = C.attend(q, k_rows, v_rows, None, [0, 3], [2], np.array([[5, -1, 3]], np.int32), page, 0.2, False, 1e5)
    assert not out.any() and np.isneginf(lse).all()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [0, 16, 48, 64])
@pytest.mark.parametrize("per_head", [False, True])
def test_norm_rotate_against_autograd(interleaved, rot, per_head):
    rng = np.random.default_rng(4)
    T, H, eps = 5, 3, 1e-3
    x = torch.from_numpy(rng.standard_normal((T, H, 64))).requires_grad_()
    g = torch.from_numpy(rng.standard_normal((H, 64) if per_head else 64)).requires_grad_()
    pos, freq = np.array([0, 3, -7, 100000, 12]), rng.random(rot // 2)
    n = torch.nn.functional.rms_norm(x, (64,), eps=eps) * g
    ang = torch.from_numpy(pos[:, None] * freq)[:, None]
    head = n[..., :rot]
    z = torch.view_as_complex((head.unflatten(-1, (-1, 2)) if interleaved
                               else head.unflatten(-1, (2, -1)).transpose(-1, -2)).contiguous()) if rot else None
    if rot:
        w = torch.view_as_real(z * torch.polar(torch.ones_like(ang), ang))
        w = w.flatten(-2) if interleaved else w.transpose(-1, -2).flatten(-2)
        y = torch.cat([w, n[..., rot:]], -1)
    else:
        y = n
    args = (x.detach().numpy(), g.detach().numpy(), pos, freq, rot, interleaved, eps)
    assert np.abs(Q.norm_rotate(*args) - y.detach().numpy()).max() < 1e-12
    dy = rng.standard_normal((T, H, 64))
    y.backward(torch.from_numpy(dy))
    dx, dg, _ = Q.norm_rotate_bwd(*args, dy)
    assert np.abs(dx - x.grad.numpy()).max() < 1e-12 and np.abs(dg - g.grad.numpy()).max() < 1e-11


def test_norm_rotate_gradient_by_differences():
    rng = np.random.default_rng(5)
    x, g = rng.standard_normal((2, 2, 64)), 1 + 0.1 * rng.standard_normal(64)
    pos, freq, dy = [4, 9], rng.random(16), rng.standard_normal((2, 2, 64))

    def f(x, g):
        return (Q.norm_rotate(x, g, pos, freq, 32, False, 1e-2) * dy).sum()

    dx, dg, _ = Q.norm_rotate_bwd(x, g, pos, freq, 32, False, 1e-2, dy)
    e, d = 1e-5, rng.standard_normal(x.shape)
    assert abs((f(x + e * d, g) - f(x - e * d, g)) / (2 * e) - (dx * d).sum()) < 1e-7
    d = rng.standard_normal(64)
    assert abs((f(x, g + e * d) - f(x, g - e * d)) / (2 * e) - (dg * d).sum()) < 1e-7
