"""Which views the bindings of the norm and of the cache take as rows, on the CPU: tensors that say they are on a GPU,
and a library that must not be reached."""
import pytest
import torch

from paper_2001_04451_amd import cache, qk


class OnGpu(torch.Tensor):
    """A CPU tensor that passes for a GPU one, as its views do."""
    is_cuda = property(lambda self: True)


def on_gpu(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


@pytest.fixture(autouse=True)
def no_library(monkeypatch):
    def refuse():
        raise AssertionError("the library was reached")
    monkeypatch.setattr(cache, "lib", refuse)
    monkeypatch.setattr(qk, "lib", refuse)


T, H, W = 6, 2, 3 * 64


def _cache():
    cfg = cache.CacheConfig(n_seq=2, T=T, H=H, Hkv=H, n_pages=4, max_pages=2, page=16, type="e4m3")
    pages = cache.Pages.empty(cfg, "cpu")
    pages = cache.Pages(*(t.as_subclass(OnGpu) for t in (pages.k, pages.v, pages.k_scale, pages.v_scale, pages.k_inv)))
    return cfg, pages, cache.Sequences(*(on_gpu(*s, dtype=torch.int32) for s in ((3,), (2,), (2, 2))))


def _one_row(*row, dtype=torch.float32):
    return on_gpu(1, *row, dtype=dtype).expand(T, *row)


def _overlapping(*row, dtype=torch.float32):
    """T rows, each 16 elements behind the last."""
    size, packed = 1, []
    for r in reversed(row):
        packed.insert(0, size)
        size *= r
    return on_gpu(size + 16 * (T - 1), dtype=dtype).as_strided((T, *row), (16, *packed))


@pytest.mark.parametrize("many", [_one_row, _overlapping])
def test_rows_that_share_storage_are_refused(many):
    """Such rows are less than their width apart; 0, taken for packed rows, would reach far past what is stored."""
    cfg, pages, seqs = _cache()
    rows = on_gpu(T, H, 64)
    for k, v in ((many(H, 64), rows), (rows, many(H, 64))):
        with pytest.raises(ValueError, match="stride"):
            cache.lsh_cache_write(cfg, pages, seqs, k, v)
        with pytest.raises(ValueError, match="stride"):
            cache.lsh_cache_read(cfg, pages, seqs, torch.float32, k, v)
    with pytest.raises(ValueError, match="stride"):
        cache.lsh_cache_attn_fwd(cfg, pages, seqs, many(H, 64, dtype=torch.bfloat16))
    c = qk.QkConfig(T=T, Hq=2, Hk=1)
    gains = (on_gpu(64), on_gpu(64), on_gpu(32))
    grads = (on_gpu(T, 2, 64), on_gpu(T, 1, 64))
    with pytest.raises(ValueError, match="stride"):
        qk.lsh_qk_norm_rotate_fwd(c, many(W), *gains)
    with pytest.raises(ValueError, match="stride"):
        qk.lsh_qk_norm_rotate_bwd(c, many(W), *gains, None, *grads)
    with pytest.raises(ValueError, match="stride"):
        qk.lsh_qk_norm_rotate_bwd(c, on_gpu(T, W), *gains, None, *grads, dx=many(W))
