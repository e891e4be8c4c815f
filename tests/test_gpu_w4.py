"""GPU parity of the 4-bit weights and the products with them with the fp64 oracle: codes, scales and values bit for bit,
products exactly where fp32 holds them and within the bound of its sums elsewhere."""
import numpy as np
import pytest
import torch

from oracle import w4 as W
from paper_2001_04451_amd import lsh, w4

from gpu_common import log

pytestmark = pytest.mark.gpu
TYPES = [("int4", 32, False), ("int4", 32, True), ("int4", 64, False), ("int4", 64, True), ("int4", 128, False),
         ("int4", 128, True), ("e2m1", 32, False)]
IDS = [f"{t}-{g}{'-zeros' if z else ''}" for t, g, z in TYPES]


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    w4.lib()
    return torch.device("cuda:0")


def config(N, K, kind):
    return w4.W4Config(N=N, K=K, type=kind[0], group=kind[1], zeros=kind[2])


def scales_tensor(scales, type_):
    t = torch.from_numpy(np.ascontiguousarray(scales))
    return t if type_ == "e2m1" else t.view(torch.int16).view(torch.bfloat16)


def pack(cfg, codes, scales, zps, gpu):
    up = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(gpu)
    return w4.lsh_w4_pack(cfg, up(W.pack_rows(codes)), scales_tensor(scales, cfg.type).to(gpu), up(zps))


def matrix(N, K, group, rng):
    """Groups of ordinary values, and some of the kinds that go wrong."""
    w = rng.standard_normal((N, K)) * np.exp(rng.standard_normal((N, 1)))
    groups = -(-K // group)
    kinds = [lambda n: np.zeros(n), lambda n: np.full(n, 7.0), lambda n: -np.abs(rng.standard_normal(n)),
             lambda n: np.abs(rng.standard_normal(n)) + 3, lambda n: (np.arange(n) % 15 - 7) + 0.5,  # borders of every code
             lambda n: rng.integers(-6, 7, n) * 1.25, lambda n: rng.standard_normal(n) * 3e38 / 5,
             lambda n: rng.standard_normal(n) * 2.0 ** -130, lambda n: np.where(np.arange(n) == 1, -0.0, 0.0),
             lambda n: rng.standard_normal(n) * 10.0 ** rng.integers(-20, 20, n)]
    for i, k in enumerate(kinds):
        n, g = (3 * i) % N, (5 * i + 1) % groups
        part = w[n, g * group:(g + 1) * group]
        part[:] = np.clip(k(len(part)), -3.3e38, 3.3e38)
    return w.astype(np.float32)


def same(got, ref):
    got, ref = got.double().cpu().numpy(), np.asarray(ref)
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    assert np.array_equal(got[~np.isnan(ref)], ref[~np.isnan(ref)])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,K", [(1, 32), (16, 128), (17, 160), (40, 416), (33, 96)])
@pytest.mark.parametrize("kind", TYPES, ids=IDS)
def test_quantize(gpu, kind, N, K, dtype):
    log("w4 quantize", kind, N, K, dtype)
    cfg = config(N, K, kind)
    w = torch.from_numpy(matrix(N, K, kind[1], np.random.default_rng(N + K))).to(dtype)
    if N > 1:
        w[1, 3], w[N // 2, K - 2], w[N - 1, 0] = float("nan"), float("inf"), -float("inf")
    codes, scales, zps = W.quantize(w.double().numpy(), *kind[:1], kind[1], kind[2])
    packed = w4.lsh_w4_quantize(cfg, w.to(gpu))
    with np.errstate(invalid="ignore"):
        ref = W.values(codes, scales, zps, kind[0], kind[1])
    same(w4.lsh_w4_unpack(cfg, packed), ref)
    # and the oracle's codes, laid out, are the same bytes
    assert torch.equal(w4.lsh_w4_unpack(cfg, pack(cfg, codes, scales, zps, gpu)).view(torch.int32)[~np.isnan(ref)],
                       w4.lsh_w4_unpack(cfg, packed).view(torch.int32)[~np.isnan(ref)])
    tiles = -(-N // 16) * -(-K // 128)
    assert torch.equal(pack(cfg, codes, scales, zps, gpu)[:tiles * 1024], packed[:tiles * 1024])


@pytest.mark.parametrize("kind", TYPES, ids=IDS)
def test_pack_and_unpack_every_code(gpu, kind):
    """Every code at every place of a tile, every scale byte; in bf16 one rounding."""
    rng = np.random.default_rng(5)
    N, K = 35, 288
    cfg = config(N, K, kind)
    groups = -(-K // kind[1])
    codes = ((np.arange(N)[:, None] * 7 + np.arange(K)) % 16).astype(np.uint8)
    if kind[0] == "e2m1":
        scales = rng.integers(0, 256, (N, groups)).astype(np.uint8)
        scales[0, :3] = [0, 254, 255]
    else:
        scales = rng.integers(0, 0x7F80, (N, groups)).astype(np.uint16)
        scales[0, :3] = [0, 1, 0x7F00]
    zps = rng.integers(0, 16, (N, groups)).astype(np.uint8) if kind[2] else None
    packed = pack(cfg, codes, scales, zps, gpu)
    with np.errstate(over="ignore", invalid="ignore"):
        ref = W.values(codes, scales, zps, kind[0], kind[1]).astype(np.float32)
    same(w4.lsh_w4_unpack(cfg, packed), ref.astype(np.float64))
    same(w4.lsh_w4_unpack(cfg, packed, torch.bfloat16), torch.from_numpy(ref).bfloat16().double().numpy())


class Exact:
    """Inputs whose products and sums fp32 holds: small whole numbers, scales of a few powers of two."""

    def __init__(self, M, N, K, kind, seed=0, stride=0):
        rng = np.random.default_rng(seed)
        groups = -(-K // kind[1])
        self.kind, self.cfg = kind, config(N, K, kind)
        self.codes = rng.integers(0, 16, (N, K)).astype(np.uint8)
        e = rng.integers(-2, 3, (N, groups))
        self.scales = (127 + e).astype(np.uint8) if kind[0] == "e2m1" else ((127 + e) << 7).astype(np.uint16)
        self.zps = rng.integers(0, 16, (N, groups)).astype(np.uint8) if kind[2] else None
        self.a = rng.integers(-3, 4, (M, K)).astype(np.float64)
        self.bias = rng.integers(-9, 10, N).astype(np.float32)
        self.resid = rng.integers(-9, 10, (M, N)).astype(np.float32)
        self.stride = stride or K

    def args(self, gpu):
        a = torch.full((len(self.a), self.stride), float("nan"), dtype=torch.bfloat16, device=gpu)
        a[:, :self.cfg.K] = torch.from_numpy(self.a).to(gpu)
        return a[:, :self.cfg.K], pack(self.cfg, self.codes, self.scales, self.zps, gpu)

    def ref(self, bias=True):
        return W.linear(self.a, self.codes, self.scales, self.zps, self.kind[0], self.kind[1],
                        self.bias.astype(np.float64) if bias else None)[0]


# (M, N, K): one row; a tile's edges in rows, outputs and inputs; inputs that end inside a tile of 128 and inside a group;
# many rows; wide and long
SIZES = [(1, 1, 32), (1, 16, 128), (2, 17, 96), (15, 33, 160), (16, 50, 1024), (17, 64, 288), (31, 48, 544), (33, 16, 2080),
         (48, 100, 256), (64, 31, 640), (65, 130, 384), (100, 257, 192), (128, 128, 512), (129, 129, 1056), (200, 96, 128),
         (257, 320, 448), (513, 65, 96), (700, 512, 1024), (1, 2047, 4128), (3, 16, 16384), (8, 4100, 64), (1, 8200, 16384), (1, 40, 12320),
         # wide calls of few rows (32 and 64 outputs a workgroup), sums split over workgroups, and the large tiles, each
         # with rows and outputs that end inside one
         (1, 8200, 160), (5, 16400, 96), (16, 16399, 64), (20, 8194, 96), (32, 16400, 288), (40, 4100, 64), (70, 200, 2112),
         (64, 130, 4128), (1000, 1050, 96), (1030, 2100, 288), (1030, 2101, 1184), (2100, 4000, 160), (2177, 4100, 544)]


@pytest.mark.parametrize("size", SIZES, ids=[f"{m}x{n}x{k}" for m, n, k in SIZES])
@pytest.mark.parametrize("kind", TYPES, ids=IDS)
def test_linear_exact(gpu, kind, size):
    """Every index, scale, zero point and tail: results equal to the last bit."""
    log("w4 linear", kind, size)
    c = Exact(*size, kind, seed=sum(size))
    a, packed = c.args(gpu)
    out = w4.lsh_linear_w4(c.cfg, a, packed)
    torch.cuda.synchronize()
    same(out, c.ref(bias=False))


@pytest.mark.parametrize("N,K", [(48, 4256), (8200, 2336), (16400, 2336)])
@pytest.mark.parametrize("kind", TYPES, ids=IDS)
def test_linear_exact_few_rows_several_turns(gpu, kind, N, K):
    """The rows kernel with 16, 32 and 64 outputs a workgroup and eight waves that each take several tiles of inputs, the
    last one ending inside: one and two tiles of rows, full and not."""
    c = Exact(32, N, K, kind, seed=N)
    a, packed = c.args(gpu)
    y = c.ref(bias=False)
    for M in (1, 16, 20, 32):
        log("w4 turns", kind, M, N, K)
        same(w4.lsh_linear_w4(c.cfg, a[:M].contiguous(), packed), y[:M])


# tiles of rows, sums joined, and the largest tiles split, with outputs stored four at a time and one by one
@pytest.mark.parametrize("M,N,K", [(1, 76, 224), (1, 77, 224), (40, 76, 224), (40, 77, 224), (300, 76, 224), (300, 77, 224),
                                   (70, 200, 2112), (70, 201, 2112), (257, 4000, 8224), (257, 4001, 8224)])
@pytest.mark.parametrize("kind", [TYPES[1], TYPES[4], TYPES[6]], ids=[IDS[1], IDS[4], IDS[6]])
def test_linear_outputs_of_every_path(gpu, kind, M, N, K):
    """Residual and its sign, in place too, relu, and what lies around the outputs."""
    log("w4 outputs of every path", kind, M, N, K)
    c = Exact(M, N, K, kind, seed=M)
    a, packed = c.args(gpu)
    assert (w4.workspace_bytes(c.cfg, M) > 0) == (K > 224)
    up = lambda t: torch.from_numpy(t).to(gpu)
    bias, resid, y = up(c.bias), up(c.resid), c.ref()
    for dtype in (torch.float32, torch.bfloat16):
        buf = torch.full((64 + M * N + 64,), 7.0, dtype=dtype, device=gpu)
        out = buf[64:64 + M * N].view(M, N)
        if dtype == torch.float32:
            for sign in (1.0, -1.0, 0.5):
                w4.lsh_linear_w4(c.cfg, a, packed, bias, resid, sign=sign, out=out)
                same(out, c.resid + sign * y)
            out.copy_(resid)
            w4.lsh_linear_w4(c.cfg, a, packed, bias, out, sign=-1.0, out=out)
            same(out, c.resid - y)
        else:
            half = torch.from_numpy(y.astype(np.float32)).bfloat16().double().numpy()
            w4.lsh_linear_w4(c.cfg, a, packed, bias, relu=True, dtype=dtype, out=out)
            same(out, np.maximum(half, 0))
        assert (buf[:64] == 7).all() and (buf[64 + M * N:] == 7).all()


def test_linear_e2m1_scales_at_both_ends(gpu):
    """The smallest scales, whose values are subnormal in bf16, and the largest whose values fp32 holds."""
    N, K = 48, 256
    cfg = config(N, K, TYPES[6])
    for low, power in ((0, 20), (246, -30)):
        for M in (1, 70):
            rng = np.random.default_rng(M)
            codes = rng.integers(0, 16, (N, K)).astype(np.uint8)
            scales = np.repeat(low + np.arange(N) % 7, K // 32).reshape(N, -1).astype(np.uint8)  # one of a row: exact sums
            a = rng.integers(-3, 4, (M, K)) * 2.0 ** power
            log("w4 ends", low, M)
            out = w4.lsh_linear_w4(cfg, torch.from_numpy(a).to(gpu).bfloat16(), pack(cfg, codes, scales, None, gpu))
            same(out, W.linear(a, codes, scales, None, "e2m1", 32)[0])


def test_quantize_at_the_end_of_fp32(gpu):
    """Magnitudes whose nearest value passes fp32's range come back infinite, the others as they should."""
    w = torch.zeros(1, 32)
    w[0, :4] = torch.tensor([3.4e38, -2.9e38, 3.5 * 2.0 ** 126, 1e38])
    step = 2.0 ** 126
    same(w4.lsh_w4_unpack(config(1, 32, TYPES[6]), w4.lsh_w4_quantize(config(1, 32, TYPES[6]), w.to(gpu)))[:, :4],
         np.array([[np.inf, -3 * step, np.inf, step]]))
    for kind in TYPES[:6]:
        cfg = config(1, 32, kind)
        with np.errstate(over="ignore"):
            ref = W.values(*W.quantize(w.double().numpy(), kind[0], kind[1], kind[2]), kind[0], kind[1]).astype(np.float32)
        same(w4.lsh_w4_unpack(cfg, w4.lsh_w4_quantize(cfg, w.to(gpu))), ref.astype(np.float64))


@pytest.mark.parametrize("kind", [TYPES[1], TYPES[4], TYPES[6]], ids=[IDS[1], IDS[4], IDS[6]])
def test_more_rows_of_tiles_than_a_grid_dimension(gpu, kind):
    """524,325 outputs: laid out, read back, quantised and multiplied past 32,768 tiles of them."""
    N, K, cut = 32_768 * 16 + 37, 96, 16_384 * 16
    log("w4 many tiles", kind)
    c = Exact(20, N, K, kind, seed=7)
    a, packed = c.args(gpu)
    with np.errstate(over="ignore", invalid="ignore"):
        same(w4.lsh_w4_unpack(c.cfg, packed), W.values(c.codes, c.scales, c.zps, kind[0], kind[1]))
    y = c.ref(bias=False)
    for M in (1, 20):
        same(w4.lsh_linear_w4(c.cfg, a[:M].contiguous(), packed), y[:M])
    w = torch.randn(N, K, generator=torch.Generator(device=gpu).manual_seed(1), device=gpu)
    whole = w4.lsh_w4_unpack(c.cfg, w4.lsh_w4_quantize(c.cfg, w))
    for part in (slice(0, cut), slice(cut, 2 * cut), slice(2 * cut, N)):
        cfg = config(len(range(N)[part]), K, kind)
        assert torch.equal(whole[part], w4.lsh_w4_unpack(cfg, w4.lsh_w4_quantize(cfg, w[part].contiguous())))


def test_packed_past_32_bits(gpu):
    """5.4 GB of codes: offsets of tiles, scales and zero points past 2^32, in every pass that takes them."""
    N, K = 82_000 + 3, 1 << 17
    for kind in (TYPES[1], TYPES[6]):
        cfg = config(N, K, kind)
        g = torch.Generator(device=gpu).manual_seed(3)
        draw = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=g, dtype=torch.uint8, device=gpu)
        codes = draw(0, 256, N, K // 2)
        e = draw(126, 129, N, K // 32)
        scales = e if kind[0] == "e2m1" else (e.short() << 7).view(torch.bfloat16)
        zps = draw(0, 16, N, K // 32) if kind[2] else None
        log("w4 past 32 bits", kind, w4.weight_bytes(cfg))
        packed = w4.lsh_w4_pack(cfg, codes, scales, zps)
        some = [0, 1, 15, 16, 20_000, 32_767, 32_768, 40_000, 65_535, 65_536, 70_001, N - 19, N - 18, N - 3, N - 1]
        part = codes[some].cpu().numpy()
        c = np.stack([part & 15, part >> 4], -1).reshape(len(some), K)
        z = None if zps is None else zps[some].cpu().numpy()
        s = scales[some].cpu()
        s = s.numpy() if kind[0] == "e2m1" else s.view(torch.int16).numpy().view(np.uint16)
        value = W.values(c, s, z, kind[0], kind[1])
        a = torch.randint(-1, 2, (200, K), generator=g, device=gpu).bfloat16()  # sums of quarters below 2^22: exact
        y = a.double().cpu().numpy() @ value.T
        for M in (1, 20, 200):
            same(w4.lsh_linear_w4(cfg, a[:M].contiguous(), packed)[:, some], y[:M])
        del codes, scales, e, zps, s, z
        w = w4.lsh_w4_unpack(cfg, packed, torch.bfloat16)
        same(w[some], value)
        w4.lsh_w4_quantize(cfg, w, packed)
        few = [0, 65_536, N - 1]
        ref = W.values(*W.quantize(w[few].double().cpu().numpy(), kind[0], kind[1], kind[2]), kind[0], kind[1])
        w = w4.lsh_w4_unpack(cfg, packed, torch.bfloat16, w)
        same(w[few], torch.from_numpy(ref).bfloat16().double().numpy())
        del packed, w


@pytest.mark.parametrize("M", [1, 20, 70, 300])
@pytest.mark.parametrize("kind", [TYPES[1], TYPES[4], TYPES[6]], ids=[IDS[1], IDS[4], IDS[6]])
def test_linear_outputs(gpu, kind, M):
    """Bias, residual and its sign, relu, both output types, rows at a stride (NaN between them), given buffers."""
    c = Exact(M, 77, 224, kind, seed=M, stride=240)
    a, packed = c.args(gpu)
    up = lambda t: torch.from_numpy(t).to(gpu)
    bias, resid, y = up(c.bias), up(c.resid), c.ref()
    log("w4 outputs", kind, M)
    same(w4.lsh_linear_w4(c.cfg, a, packed, bias), y)
    same(w4.lsh_linear_w4(c.cfg, a, packed, bias, resid, sign=-1.0), c.resid - y)
    same(w4.lsh_linear_w4(c.cfg, a, packed, bias, resid, sign=0.5), c.resid + 0.5 * y)
    half = lambda t: torch.from_numpy(t.astype(np.float32)).bfloat16().double().numpy()
    same(w4.lsh_linear_w4(c.cfg, a, packed, bias, dtype=torch.bfloat16), half(y))
    out = torch.full((M + 2, 77), 7.0, dtype=torch.bfloat16, device=gpu)
    # rows beside the result are left alone (an odd number of outputs: the middle starts off any alignment but its own)
    buf = torch.full((64 + M * 77 + 64,), 7.0, dtype=torch.bfloat16, device=gpu)
    got = w4.lsh_linear_w4(c.cfg, a, packed, bias, relu=True, dtype=torch.bfloat16, out=buf[64:64 + M * 77].view(M, 77))
    same(got, np.maximum(half(y), 0))
    assert (buf[:64] == 7).all() and (buf[64 + M * 77:] == 7).all() and (out == 7).all()


@pytest.mark.parametrize("kind", [TYPES[1], TYPES[4], TYPES[6]], ids=[IDS[1], IDS[4], IDS[6]])
def test_linear_exact_split_large_tiles(gpu, kind):
    """The largest tiles with their inputs split: rows, outputs and inputs that end inside one."""
    log("w4 split large", kind)
    c = Exact(257, 4000, 8224, kind, seed=5)
    a, packed = c.args(gpu)
    y = c.ref()
    bias = torch.from_numpy(c.bias).to(gpu)
    same(w4.lsh_linear_w4(c.cfg, a, packed, bias), y)
    same(w4.lsh_linear_w4(c.cfg, a, packed, bias, dtype=torch.bfloat16),
         torch.from_numpy(y.astype(np.float32)).bfloat16().double().numpy())


@pytest.mark.parametrize("size", [(66, 8, 256), (130, 72, 224), (130, 200, 1184), (513, 2056, 96), (1030, 2104, 288), (2100, 4024, 160)],
                         ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("kind", [TYPES[1], TYPES[4], TYPES[6]], ids=[IDS[1], IDS[4], IDS[6]])
def test_linear_bf16_rows(gpu, kind, size):
    """bf16 results of a number of outputs that is a multiple of 8, in every size of tiles, with bias and relu, and what
    lies behind them."""
    log("w4 bf16 rows", kind, size)
    M, N, K = size
    c = Exact(M, N, K, kind, seed=N)
    a, packed = c.args(gpu)
    y = torch.from_numpy(c.ref().astype(np.float32)).bfloat16().double().numpy()
    bias = torch.from_numpy(c.bias).to(gpu)
    buf = torch.full((M * N + 128,), 7.0, dtype=torch.bfloat16, device=gpu)
    out = buf[64:64 + M * N].view(M, N)
    same(w4.lsh_linear_w4(c.cfg, a, packed, bias, dtype=torch.bfloat16, out=out), y)
    same(w4.lsh_linear_w4(c.cfg, a, packed, bias, relu=True, dtype=torch.bfloat16, out=out), np.maximum(y, 0))
    assert (buf[:64] == 7).all() and (buf[64 + M * N:] == 7).all()


@pytest.mark.parametrize("M", [1, 16, 61, 130, 400])
@pytest.mark.parametrize("kind", TYPES, ids=IDS)
def test_linear_real(gpu, kind, M):
    """Weights as quantised, rows as activations.  Codes are exact in the products; a sum of K of them and of the groups'
    scaled sums takes at most K + 4 groups roundings of what is there, which `size` bounds."""
    rng = np.random.default_rng(M)
    N, K = 200, 1184
    cfg = config(N, K, kind)
    w = (rng.standard_normal((N, K)) * np.exp(0.3 * rng.standard_normal((N, 1)))).astype(np.float32)
    codes, scales, zps = W.quantize(w, *kind[:1], kind[1], kind[2])
    a = torch.from_numpy((rng.standard_normal((M, K)) * np.exp(0.5 * rng.standard_normal(K))).astype(np.float32)).bfloat16()
    ref, size = W.linear(a.double().numpy(), codes, scales, zps, kind[0], kind[1])
    log("w4 real", kind, M)
    packed = w4.lsh_w4_quantize(cfg, torch.from_numpy(w).to(gpu))
    out = w4.lsh_linear_w4(cfg, a.to(gpu), packed)
    err = np.abs(out.double().cpu().numpy() - ref)
    assert (err <= (K + 4 * cfg.groups() + 8) * 2.0 ** -24 * size).all()
    # over all outputs together: roundings of either sign do not add up to a tenth of their sum's bound
    assert np.linalg.norm(err) <= 0.1 * (K + 4 * cfg.groups() + 8) * 2.0 ** -24 * np.linalg.norm(size)
    b16 = w4.lsh_linear_w4(cfg, a.to(gpu), packed, dtype=torch.bfloat16)
    assert torch.equal(b16, out.bfloat16())
    assert torch.equal(w4.lsh_linear_w4(cfg, a.to(gpu), packed), out)  # bit for bit again


@pytest.mark.parametrize("M", [3, 90])
@pytest.mark.parametrize("kind", [TYPES[5], TYPES[6]], ids=[IDS[5], IDS[6]])
def test_linear_nan_stays_where_it_is(gpu, kind, M):
    """A group that is NaN spoils its output alone, a row that is NaN its row alone."""
    c = Exact(M, 40, 320, kind, seed=9)
    c.scales[11, 1] = 255 if kind[0] == "e2m1" else 0x7FC0
    c.a[2, 300] = np.nan
    log("w4 nan", kind, M)
    a, packed = c.args(gpu)
    out = w4.lsh_linear_w4(c.cfg, a, packed).double().cpu().numpy()
    bad = np.zeros(out.shape, bool)
    bad[2], bad[:, 11] = True, True
    assert np.isnan(out[bad]).all()
    c.scales[11, 1], c.a[2, 300] = (127 if kind[0] == "e2m1" else 127 << 7), 0
    assert np.array_equal(out[~bad], c.ref(bias=False)[~bad])


def test_linear_large_values(gpu):
    """Activations and scales far apart: sums of up to 2^120 and down to 2^-100 keep their bits."""
    for kind in (TYPES[4], TYPES[6]):
        c = Exact(5, 32, 256, kind, seed=2)
        for power in (90, -90):
            a, packed = c.args(gpu)
            out = w4.lsh_linear_w4(c.cfg, (a.float() * 2.0 ** power).bfloat16().contiguous(), packed)
            same(out, c.ref(bias=False) * 2.0 ** power)


@pytest.mark.parametrize("M", [1, 40, 260, 90])
def test_linear_streams_and_graphs(gpu, M):
    """On another stream, two at once with a workspace each, and captured and replayed over changing rows with eager calls
    between."""
    c = Exact(M, 96, 640 if M != 90 else 2144, TYPES[3], seed=4)  # 90 rows: split sums, joined through the workspace
    assert (w4.workspace_bytes(c.cfg, M) > 0) == (M == 90)
    a, packed = c.args(gpu)
    a = a.contiguous()
    ref = c.ref(bias=False)
    log("w4 streams", M)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    torch.cuda.synchronize()
    for s in streams:
        with torch.cuda.stream(s):
            outs.append(w4.lsh_linear_w4(c.cfg, a, packed, workspace=w4.workspace(c.cfg, M, gpu)))
    torch.cuda.synchronize()
    for o in outs:
        same(o, ref)
    ws = w4.workspace(c.cfg, M, gpu)
    ws.fill_(255)
    out = torch.empty(M, 96, device=gpu)
    g = torch.cuda.CUDAGraph()
    rows = a.clone()
    with torch.cuda.graph(g):
        w4.lsh_linear_w4(c.cfg, rows, packed, out=out, workspace=ws)
    for k in (1, 2, 3):
        rows.copy_(a * k)
        ws.fill_(k)
        out.fill_(float("nan"))
        g.replay()
        eager = w4.lsh_linear_w4(c.cfg, rows, packed)
        torch.cuda.synchronize()
        same(out, k * ref)
        assert torch.equal(eager, out)


def test_linear_rows_far_apart(gpu):
    """Rows 2^24 elements apart: offsets past 32 bits."""
    c = Exact(70, 40, 160, TYPES[3], seed=8)
    a, packed = c.args(gpu)
    far = torch.empty(70 << 24, dtype=torch.bfloat16, device=gpu).view(70, 1 << 24)
    far[:, :160].copy_(a)
    far[:, 160:320] = float("nan")
    log("w4 far rows")
    same(w4.lsh_linear_w4(c.cfg, far[:, :160], packed), c.ref(bias=False))
    near = torch.empty(70 << 22, dtype=torch.bfloat16, device=gpu).view(70, 1 << 22)
    near[:, :160].copy_(a)
    near[:, 160:320] = float("nan")
    same(w4.lsh_linear_w4(c.cfg, near[:, :160], packed), c.ref(bias=False))


def test_bf16_products_of_the_same_weights(gpu):
    """e2m1 weights are exact in bf16: the bf16 product of the unpacked matrix gives the same results."""
    c = Exact(96, 128, 256, TYPES[6], seed=6)
    a, packed = c.args(gpu)
    w = w4.lsh_w4_unpack(c.cfg, packed, torch.bfloat16)
    assert torch.equal(lsh.linear_bf16(a.contiguous(), w), w4.lsh_linear_w4(c.cfg, a, packed))


def test_refused_rows(gpu):
    cfg = config(16, 64, TYPES[0])
    packed = w4.lsh_w4_quantize(cfg, torch.ones(16, 64, device=gpu))
    with pytest.raises(lsh.LshError):  # rows at a stride that is no multiple of 8
        w4.lsh_linear_w4(cfg, torch.zeros(4, 68, dtype=torch.bfloat16, device=gpu)[:, :64], packed)
    with pytest.raises(lsh.LshError):  # rows that do not start on 16 bytes
        w4.lsh_linear_w4(cfg, torch.zeros(4, 72, dtype=torch.bfloat16, device=gpu)[:, 1:65], packed)
    with pytest.raises(lsh.LshError):
        w4.lsh_linear_w4(cfg, torch.zeros(4, 64, dtype=torch.bfloat16, device=gpu), packed, relu=True)
