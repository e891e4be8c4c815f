"""Sequences without new tokens beside those that have some, as a captured step with free places has them (one MI355X)."""
import numpy as np
import pytest
import torch

from paper_2001_04451_amd import cache

from gpu_common import log
from test_gpu_cache import Case, _check_pages, _expect, _write, check_attention, gpu  # noqa: F401

pytestmark = pytest.mark.gpu


def _cases():
    rng = np.random.default_rng(81)
    for n_seq, active, new in ((3000, 40, 1), (700, 25, 11), (130, 1, 1), (2000, 2000, 1), (16384, 9, 3)):
        news = np.zeros(n_seq, int)
        news[rng.choice(n_seq, active, replace=False)] = rng.integers(1, new + 1, active)
        yield n_seq, active, news, np.where(news > 0, news + rng.integers(0, 30, n_seq), rng.integers(0, 3, n_seq))


@pytest.mark.parametrize("i", range(5))
def test_idle_sequences(gpu, i):  # noqa: F811
    n_seq, active, news, lens = list(_cases())[i]
    c = Case("e4m3", True, 1, 1, 16, lens, news, seed=82)
    log("cache idle sequences", n_seq, active)
    k, v = (torch.from_numpy(c.rng.standard_normal((c.T, 1, 64)).astype(np.float32)) for _ in "kv")
    pages = _write(c, gpu, k, v)
    _check_pages(pages, _expect(c, k.double().numpy(), v.double().numpy()))
    rk, rv = cache.lsh_cache_read(c.cfg, pages, c.seqs(gpu), torch.float32)
    assert ((rv - v.to(gpu)).abs() <= 2.0 ** -4 * v.to(gpu).abs().clamp(min=2.0 ** -5)).all()
    check_attention(c, gpu)


def test_idle_sequences_joined_by_sixteen_lanes(gpu):  # noqa: F811
    """Few long sequences among many idle ones, rows enough for joins of several rows a wave."""
    rng = np.random.default_rng(83)
    news, lens = np.zeros(2500, int), rng.integers(0, 4, 2500)
    at = rng.choice(2500, 300, replace=False)
    news[at], lens[at] = 7, 30
    lens[at[:6]] = rng.integers(900, 2500, 6)
    log("cache idle sequences joined")
    check_attention(Case("bf16", False, 8, 2, 16, lens, news, seed=84), gpu)
