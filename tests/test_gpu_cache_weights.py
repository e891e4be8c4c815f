"""Attention of long calls (2^24 query-key pairs and more by the table's width) keeps 16 bits of its weights where tiles have
16 or 64 rows, whole prompts aside (one MI355X)."""
import numpy as np
import pytest

from oracle import cache as C
from paper_2001_04451_amd import cache

from gpu_common import log
from test_gpu_cache import TYPES, Case, gpu  # noqa: F401
from test_gpu_cache_tiles import tiles, widen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("what", ["few tokens", "chunks"])
@pytest.mark.parametrize("shared", [True, False])
@pytest.mark.parametrize("type_", TYPES)
def test_weights_of_long_calls_keep_sixteen_bits(gpu, type_, shared, what):  # noqa: F811
    """A weight is off by 2^-16 of it at most (what its bf16 rounding leaves, itself at most 2^-8 of it, is rounded to
    bf16 once more); the sums of up to 700 keys take fewer than 700 roundings of 2^-24 to fp32.  Products, sum and
    division together: (2^-16 + 700 2^-24) twice, below 2^-12, and the output's own rounding of 2^-8."""
    if what == "few tokens":
        c = Case(type_, shared, 8 if not shared else 4, 4, 32, [1, 60, 333, 700], [1, 2, 1, 3], seed=21)
        widen(c, 6, 1 << 24)
    else:
        c = tiles(Case(type_, shared, 4, 4 if shared else 2, 32, [300, 700], [70, 40], seed=22), 64)
    host, kr, vr = c.host_pages()
    log("cache attention precision of long calls", type_, shared, what)
    out, _ = cache.lsh_cache_attn_fwd(c.cfg, c.pages(host, gpu), c.seqs(gpu), c.q.to(gpu))
    inv = None if host[4] is None else host[4].astype(np.float64)
    ref, _, spread, _ = C.attend(c.q.double().numpy(), kr, vr, inv, c.first, c.lens, c.table, c.page, 0.125, c.shared,
                                 c.cfg.self_mask)
    # a logit's 64 products are at most |q||k|/8 together: 70 roundings of that in fp32, and twice for numerator and sum
    longest = 1 if shared else np.linalg.norm(kr, axis=-1).max()
    dz = 2 * 70 * 2.0 ** -24 * np.linalg.norm(c.q.double().numpy(), axis=-1, keepdims=True) * 0.125 * longest
    tol = (2.0 ** -12 + dz) * spread + 2.0 ** -8 * np.abs(ref)
    err = np.abs(out.double().cpu().numpy() - ref)
    assert (err <= tol).all(), f"{(err / np.maximum(tol, 1e-300)).max():.2f} of the tolerance"
