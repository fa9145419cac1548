"""PagedKVCache's bookkeeping on the host, with the library's calls replaced: what a step or an eviction that fails leaves behind."""
import pytest
import torch

from paper_2502_00425_b200 import binding as B
from paper_2502_00425_b200 import kvcache as KC


class Handle:
    def __init__(self, K, V, k_scale=None, v_scale=None):
        self.n_kv_heads, self.head_dim, self.page_size, self.device = K.shape[1], K.shape[3], K.shape[2], K.device


@pytest.fixture
def make(monkeypatch):
    monkeypatch.setattr(B, "KVCache", Handle)
    monkeypatch.setattr(B, "mq_last_device_status", lambda ws: (B.MQ_OK, 0))
    return lambda *args, **kw: KC.PagedKVCache(*args, device="cpu", **kw)


def _state(cache):
    return (list(cache.free), [list(p) for p in cache.pages], list(cache.lengths), list(cache.tokens))


def _refuse(*args, **kw):
    raise B.MqError(B.MQ_ERR_INVALID_ARG, "mq_kv_evict")


def test_a_refused_eviction_keeps_its_pages(make, monkeypatch):
    cache = make(2, 12, 64, 2, 64, page_size=16)
    cache.track_weights()
    cache.extend([40, 20])
    before, weights = _state(cache), cache.weights.clone()
    monkeypatch.setattr(B, "mq_kv_evict", _refuse)
    for _ in range(5):                       # (the pool has room for two evictions' pages)
        with pytest.raises(B.MqError):
            cache.evict(30, 20, 20)
        assert _state(cache) == before and torch.equal(cache.weights, weights)
    with pytest.raises(RuntimeError):        # no memory for the outputs: nothing of the library was called yet
        monkeypatch.setattr(KC.torch, "zeros", lambda *a, **k: (_ for _ in ()).throw(RuntimeError("out of memory")))
        cache.evict(30, 2, 2)
    assert _state(cache) == before


def test_an_eviction_moves_to_fresh_pages_and_frees_the_old_ones(make, monkeypatch):
    calls = []
    monkeypatch.setattr(B, "mq_kv_evict", lambda *a, **k: calls.append(a))
    cache = make(2, 10, 64, 2, 64, page_size=16)
    cache.track_weights()
    cache.extend([40, 20])
    old = [list(p) for p in cache.pages]
    cache.evict(24, 2, 2)
    assert cache.lengths == [24, 20] and cache.tokens == [40, 20] and len(calls) == 1
    assert [len(p) for p in cache.pages] == [2, 2] and not set(sum(cache.pages, [])) & set(sum(old, []))
    assert sorted(cache.free + sum(cache.pages, [])) == list(range(10))
    for b in range(2):
        assert cache.table[b, :2].tolist() == cache.pages[b] and bool((cache.table[b, 2:] == -1).all())


def test_an_extension_that_fails_changes_nothing(make, monkeypatch):
    cache = make(2, 12, 100, 2, 64, page_size=16)
    cache.extend([40, 20])
    before = _state(cache)
    for name, at in (("tensor", 1), ("tensor", 3), ("tensor", 5), ("full", 1), ("full", 2)):
        real, count = getattr(torch, name), [0]

        def fails(*args, **kw):
            count[0] += 1
            if count[0] == at:
                raise RuntimeError("out of memory")
            return real(*args, **kw)

        with monkeypatch.context() as m:
            m.setattr(KC.torch, name, fails)
            with pytest.raises(RuntimeError, match="out of memory"):
                cache.extend([30, 30])
        assert _state(cache) == before
    step = cache.extend([30, 30])
    assert cache.lengths == [70, 50] and step.kv_len.tolist() == [70, 50] and step.total == 60


def test_a_step_is_undone(make):
    cache = make(3, 12, 100, 2, 64, page_size=16)
    first = cache.extend([40, 16, 0])
    before = _state(cache)
    for new in ([1, 1, 1], [30, 0, 17], [8, 8, 8], [0, 0, 1]):
        step = cache.extend(new)
        arrays = [step.cu_q, step.kv_len, step.slots, step.pos]
        cache.undo(step)
        assert _state(cache) == before
        again = cache.extend(new)            # the same pages and positions
        assert all(torch.equal(a, b) for a, b in zip(arrays, [again.cu_q, again.kv_len, again.slots, again.pos]))
        for b in range(3):
            n = len(cache.pages[b])
            assert cache.table[b, :n].tolist() == cache.pages[b]
        with pytest.raises(RuntimeError):
            cache.undo(step)                 # not the last one
        cache.undo(again)
        with pytest.raises(RuntimeError):
            cache.undo(again)
    with pytest.raises(RuntimeError):
        cache.undo(first)
    assert _state(cache) == before


def test_a_step_is_not_undone_behind_an_eviction(make, monkeypatch):
    monkeypatch.setattr(B, "mq_kv_evict", lambda *a, **k: None)
    cache = make(1, 10, 64, 2, 64, page_size=16)
    cache.track_weights()
    step = cache.extend([40])
    cache.evict(40, 0, 0)
    with pytest.raises(RuntimeError):
        cache.undo(step)
    assert cache.lengths == [40]


def test_a_cache_stays_on_the_device_it_was_made_on(make, monkeypatch):
    """Not on whichever is current when a step's arrays are made, or when its status is read."""
    cache = make(1, 10, 64, 2, 64, page_size=16)
    assert cache.device == cache.K.device == cache.table.device and isinstance(cache.device, torch.device)
    seen = []

    class Current:
        def __init__(self, tensor):
            self.tensor = tensor

        def __enter__(self):
            seen.append(self.tensor)

        def __exit__(self, *exc):
            seen.append(None)

    monkeypatch.setattr(KC.torch.cuda, "device_of", Current)
    monkeypatch.setattr(B, "mq_last_device_status", lambda ws: (B.MQ_OK if seen and seen[-1] is ws else B.MQ_ERR_CUDA, 0))
    assert cache.status_ok()
