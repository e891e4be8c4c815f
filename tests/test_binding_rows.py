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


def test_one_row_has_any_stride():
    """With one token nothing lies a stride away: a configuration that names one for its batches takes a single row, which
    is passed with that stride, and a view's own does not matter."""
    fused = on_gpu(4, 12 * 64)
    cfg = cache.CacheConfig(n_seq=1, T=1, H=4, Hkv=4, n_pages=1, max_pages=1, q_stride=768)
    row = fused[:1, 256:512].unflatten(1, (4, 64))
    dev = row.device
    assert cache._rows(row, cfg, 4, "q", cfg.q_stride, dev) == 768
    assert cache._rows(on_gpu(1, 4, 64), cfg, 4, "q", cfg.q_stride, dev) == 768
    assert cache._rows(row, cfg, 4, "k", cfg.k_stride, dev) == 0
    assert qk._token_rows(fused[:1], 1, 256, "x", 768) == 768
    assert qk._token_rows(fused[:1, :256], 1, 256, "x", 512) == 512
    assert qk._token_rows(fused[:1], 1, 256, "x", 0) == 0


def test_strides_of_many_rows():
    """Packed rows, views with their own stride, and one that is not what the configuration says."""
    fused = on_gpu(T, 12 * 64)
    cfg, *_ = _cache()
    view, packed = fused[:, 128:256].unflatten(1, (2, 64)), on_gpu(T, 2, 64)
    dev = view.device
    assert cache._rows(view, cfg, 2, "k", 0, dev) == cache._rows(view, cfg, 2, "k", 768, dev) == 768
    assert cache._rows(packed, cfg, 2, "k", 0, dev) == 0 and cache._rows(packed, cfg, 2, "k", 128, dev) == 128
    assert qk._token_rows(fused, T, 256, "x", 0) == qk._token_rows(fused, T, 256, "x", 768) == 768
    assert qk._token_rows(on_gpu(T, W), T, W, "x", 0) == 0 and qk._token_rows(on_gpu(T, W), T, W, "x", W) == W
    for rows in (lambda: cache._rows(view, cfg, 2, "k", 256, dev), lambda: qk._token_rows(fused, T, 256, "x", 256)):
        with pytest.raises(ValueError, match="the configuration"):
            rows()


def test_workspaces_are_device_memory():
    """A workspace on the host, on another device than the tensors, or of less storage than elements never reaches the library."""
    cfg, pages, seqs = _cache()
    q, out, lse = on_gpu(T, H, 64, dtype=torch.bfloat16), on_gpu(T, H, 64, dtype=torch.bfloat16), on_gpu(T, H)
    c = qk.QkConfig(T=T, Hq=2, Hk=1)
    args = (c, on_gpu(T, W), on_gpu(64), on_gpu(64), on_gpu(32), None, on_gpu(T, 2, 64), on_gpu(T, 1, 64), on_gpu(T, W))
    large = 1 << 20
    host = torch.zeros(large, dtype=torch.uint8)
    elsewhere = torch.zeros(large, dtype=torch.uint8, device="meta").as_subclass(OnGpu)
    for bad in (host, elsewhere, on_gpu(1, dtype=torch.uint8).expand(large), on_gpu(large, dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError, match="workspace"):
            cache.lsh_cache_attn_fwd(cfg, pages, seqs, q, out=out, lse=lse, workspace=bad)
        with pytest.raises(ValueError, match="workspace"):
            qk.lsh_qk_norm_rotate_bwd(*args, workspace=bad)


def test_sequences_are_checked_for_each_device():
    """One set of sequences and one configuration, over pools of two devices."""
    cfg, _, seqs = _cache()
    seqs.check(cfg, torch.device("cpu"))
    with pytest.raises(ValueError, match="first is on cpu"):
        seqs.check(cfg, torch.device("cuda:1"))
    seqs.check(cfg, torch.device("cpu"))
