"""Attention over the cache at the ends of the documented range of values and of the logits for which no running maximum
is taken (one MI355X)."""
import numpy as np
import pytest

from paper_2001_04451_amd import cache  # noqa: F401

from gpu_common import log
from test_gpu_cache import Case, check_attention, gpu  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("exponent", [60, -60])
@pytest.mark.parametrize("bound", [29.9, 30.1, 59.5])
@pytest.mark.parametrize("type_", ["bf16", "e4m3"])
@pytest.mark.parametrize("shape", [([4000], [1]), ([4000, 9], [20, 1]), ([3000], [300])])
def test_large_logits_times_large_values(gpu, shape, type_, bound, exponent):  # noqa: F811
    """Keys along the queries, whose logits are all as large (small, against every second query) as the queries' length
    lets them be: 2^bound, and values near 2^exponent.  The output is a mean of the values, whatever the weights' size."""
    lens, news = shape
    c = Case(type_, True, 2, 2, 16, lens, news, seed=31)
    u = c.rng.standard_normal(64)
    c.k[:] = u
    c.v = np.ldexp(1 + c.rng.random(c.v.shape), exponent).astype(np.float32)
    q = u / np.linalg.norm(u) * bound / (0.125 * np.log2(np.e))
    sign = np.where(np.arange(c.T) % 2 == 0, 1, -1)[:, None, None]
    c.q[:] = c.q.new_tensor(q * sign)
    log("cache attention range", shape, type_, bound, exponent)
    check_attention(c, gpu)
