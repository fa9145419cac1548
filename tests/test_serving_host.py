"""Host-side checks (no GPU) of the calls around a serving step: refusals before anything is enqueued, and pins of their oracle."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import kv_oracle as O
from oracle import plan_oracle as P
from oracle import sample_oracle as S
from paper_2502_00425_b200 import binding as B
from paper_2502_00425_b200 import build
from paper_2502_00425_b200 import kvcache as KC

A = 0x10000   # a fake, aligned device address: validation must come before it is used


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return B.load()


def _cache(K=A, V=A, page_stride=4 * 64 * 128, head_stride=64 * 128, slot_stride=128, n_pages=10, page=64, hkv=4, dim=128, flags=0,
           ks=None, vs=None):
    return B.mq_kv_cache(K, V, page_stride, head_stride, slot_stride, n_pages, page, hkv, dim, flags, ks, vs)


# ------------------------------------------------------------------------------------------------ rotary embedding
def test_rotary_refusals(lib):
    theta = (C.c_double * 64)(*[0.5] * 64)
    rope = lambda rot=64, flags=0, amp=1.0, theta=theta: B.mq_rope(C.cast(theta, C.POINTER(C.c_double)) if theta else None, rot, flags, amp)

    def call(r=None, T=5, hq=8, hkv=4, dim=128, eps=1e-6, q=A, ldq=1024, pos=A, qo=A, slots=A, cache=None, none=False):
        r = rope() if r is None else r
        return lib.mq_qk_norm_rope_scaled(q, ldq, A, hkv * dim, A, hkv * dim, T, hq, hkv, dim, None, None, eps, pos, None if none else C.byref(r),
                                          qo, hq * dim, None, 0, C.byref(cache or _cache()), slots, None)

    assert call(none=True) == B.MQ_ERR_INVALID_ARG
    assert call(rope(rot=-8)) == call(rope(rot=136)) == call(rope(flags=2)) == call(rope(theta=None)) == B.MQ_ERR_INVALID_ARG
    assert call(rope(rot=68)) == B.MQ_ERR_UNSUPPORTED
    for bad in (math.nan, math.inf, -2e6):
        assert call(rope(theta=(C.c_double * 64)(*[0.5] * 31 + [bad] + [0.5] * 32))) == B.MQ_ERR_INVALID_ARG
    assert call(rope(rot=32, theta=(C.c_double * 64)(*[0.5] * 31 + [math.nan] + [0.5] * 32)), q=None) == B.MQ_ERR_INVALID_ARG
    assert call(rope(amp=math.inf)) == call(rope(amp=math.nan)) == call(eps=-1.0) == call(T=-1) == call(hq=0) == B.MQ_ERR_INVALID_ARG
    assert call(dim=96) == B.MQ_ERR_UNSUPPORTED
    assert call(q=None) == call(pos=None) == call(qo=None) == call(slots=None) == call(ldq=512) == B.MQ_ERR_INVALID_ARG
    assert call(q=A + 2) == call(ldq=1028) == B.MQ_ERR_ALIGNMENT
    assert call(cache=_cache(dim=64)) == call(cache=_cache(hkv=2)) == B.MQ_ERR_INVALID_ARG
    assert call(T=0) == call(rope(rot=0, theta=None), T=0) == B.MQ_OK


def test_frequencies_of_the_binding():
    for kw in (dict(), dict(factor=4.0), dict(factor=4.0, original=32768), dict(factor=2.0, original=100, fast=8.0, slow=2.0)):
        got = np.array(B.Rope(64, **kw).theta)
        want = O.rope_theta(64, 10000.0, **kw)
        assert np.all(np.abs(got - want) <= 2.0 ** -48 * want)
    by_parts, plain = B.Rope(128, factor=8.0, original=4096).theta, B.Rope(128).theta
    assert by_parts[0] == plain[0] and by_parts[-1] == plain[-1] / 8.0       # many turns: kept; less than one: divided
    assert all(p / 8.0 <= t <= p for t, p in zip(by_parts, plain))
    assert B.Rope(4, theta=[1, 2]).theta == [1.0, 2.0]
    for bad in (dict(rotary_dim=7), dict(rotary_dim=-2), dict(rotary_dim=8, theta=[1.0]), dict(rotary_dim=8, base=0.5),
                dict(rotary_dim=8, factor=0.0), dict(rotary_dim=8, original=4096, fast=1.0, slow=1.0)):
        with pytest.raises(ValueError):
            B.Rope(**bad)


def test_rotary_oracle_reduces_to_the_whole_head():
    rng = np.random.default_rng(0)
    x, pos, gain = rng.standard_normal((5, 3, 16)), np.arange(5) * 7, rng.standard_normal(16)
    for half in (False, True):
        y, mag = O.norm_rope(x, gain, 1e-6, pos, 10000.0, half)
        y2, mag2 = O.norm_rope_scaled(x, gain, 1e-6, pos, O.rope_theta(16, 10000.0), half, 1.0)
        assert np.allclose(y, y2, rtol=0, atol=1e-13) and np.allclose(mag, mag2, rtol=1e-13)
        y3, _ = O.norm_rope_scaled(x[..., :8], None, 0, pos, O.rope_theta(8, 10000.0), half, 2.0)
        y4, _ = O.norm_rope_scaled(x, None, 0, pos, O.rope_theta(8, 10000.0), half, 2.0)
        assert np.array_equal(y3, y4[..., :8]) and np.array_equal(y4[..., 8:], x[..., 8:])


# ------------------------------------------------------------------------------------------------ sampling
def test_sample_refusals(lib):
    def call(x=A, ld=1000, n=4, v=1000, flags=1, t=A, u=A, token=A):
        return lib.mq_sample(x, ld, n, v, flags, t, None, None, None, u, token, None, None, None)

    assert call(n=-1) == call(v=0) == call(v=-5) == call(ld=999) == call(flags=2) == B.MQ_ERR_INVALID_ARG
    assert call(x=None) == call(t=None) == call(u=None) == call(token=None) == B.MQ_ERR_INVALID_ARG
    assert call(v=(1 << 20) + 1, ld=1 << 21) == call(n=(1 << 24) + 1) == B.MQ_ERR_UNSUPPORTED
    assert call(x=A + 2) == call(x=A + 1, flags=0) == B.MQ_ERR_ALIGNMENT
    assert call(n=0) == call(n=0, x=None) == B.MQ_OK


def test_sample_oracle_by_hand():
    x = np.log([4.0, 2.0, 1.0, 1.0])
    for u, want in ((0.0, 0), (0.49, 0), (0.5, 1), (0.74, 1), (0.75, 2), (0.88, 3)):
        assert S.sample(x, 1.0, u)[0] == want
    assert S.sample(x, 1.0, 0.6, top_k=2)[2].tolist() == [0, 1] and S.sample(x, 1.0, 0.7, top_k=2)[0] == 1
    assert S.sample(x, 1.0, 0.0, top_p=0.5)[2].tolist() == [0]               # exactly half lies before the second
    assert S.sample(x, 1.0, 0.0, top_p=0.51)[2].tolist() == [0, 1] and S.sample(x, 1.0, 0.0, top_p=0.9)[2].tolist() == [0, 1, 2, 3]
    assert S.sample(x, 1.0, 0.0, top_k=2, top_p=0.7)[2].tolist() == [0, 1]   # of the first two, two thirds lie before the second
    assert S.sample(x, 1.0, 0.0, top_k=2, top_p=0.6)[2].tolist() == [0]
    assert S.sample(x, 0.5, 0.0, min_p=0.25)[2].tolist() == [0, 1]           # weights 1, 1/4, 1/16
    assert S.sample(np.array([1.0, 3.0, 3.0]), 0.0, 0.9)[0] == 1
    assert S.sample(np.array([np.nan, -np.inf]), 1.0, 0.9)[0] == -1
    assert abs(S.sample(x, 1.0, 0.5)[1] - np.log(0.25)) < 1e-15


# ------------------------------------------------------------------------------------------------ bookkeeping
def test_plan_refusals(lib):
    def call(n=4, width=7, page=64, pages=100, kv=A, seen=A, table=A, borrowed=None, free=A, n_free=A, new=A, keep=None, rows=10, cu=A, slots=A,
             pos=A, none=False):
        s = B.mq_kv_state(n, width, page, pages, kv, seen, table, borrowed, free, n_free)
        return lib.mq_kv_plan(None if none else C.byref(s), new, keep, rows, cu, slots, pos, None, None)

    assert call(none=True) == call(n=-1) == call(width=-1) == call(pages=-1) == call(rows=-1) == call(page=0) == B.MQ_ERR_INVALID_ARG
    assert call(n=2049) == call(width=(1 << 22) + 1) == call(page=48) == call(page=8) == call(page=512) == call(rows=(1 << 30) + 1) == B.MQ_ERR_UNSUPPORTED
    for name in ("kv", "seen", "table", "free", "n_free", "new", "cu", "slots", "pos"):
        assert call(**{name: None}) == B.MQ_ERR_INVALID_ARG


def test_plan_oracle_by_hand():
    state = dict(kv_len=[5, 0], seen=[9, 0], borrowed=[0, 0], table=[[3, 5, -1], [-1, -1, -1]], free=[4, 2, 1, 0], n_pages=6)
    assert P.plan(state, [4, 3], None, 8, 4) == ([0, 4, 7], [21, 22, 23, 0, 4, 5, 6, -1], [9, 10, 11, 12, 0, 1, 2, 0])
    assert state["table"] == [[3, 5, 0], [1, -1, -1]] and state["free"] == [4, 2] and state["kv_len"] == [9, 3]
    assert P.plan(state, [0, 0], [5, 0], 0, 4) == ([0, 0, 0], [], [])
    assert state["free"] == [4, 2, 1, 0] and state["seen"] == [9, 0]
    state["borrowed"] = [1, 0]
    assert P.plan(state, [1, 0], [0, 0], 1, 4) == ([0, 1, 1], [20], [0])      # its own page 5 goes back and comes again; page 3 is not its own
    assert state["free"] == [4, 2, 1, 0] and state["borrowed"] == [0, 0]
    with pytest.raises(P.Refused):
        P.plan(state, [12, 12], None, 24, 4)


# ------------------------------------------------------------------------------------------------ attention behind a shared prefix
def test_shared_attention_refusals(lib):
    def call(q=A, ldq=1024, hq=8, scale=0.1, o=A, ldo=1024, ws=A, wsb=1 << 40, leader=A, shared=A, cache=None, n_seq=2, total=5, max_q=4,
             max_pages=7, cu=A, kv=A, table=A):
        b = B.mq_kv_batch(n_seq, total, max_q, max_pages, cu, kv, table, None)
        return lib.mq_kv_attention_shared(q, ldq, C.byref(b), leader, shared, C.byref(cache or _cache()), hq, scale, o, ldo, None, ws, wsb, None)

    assert call(n_seq=-1) == call(max_q=6) == call(cu=None) == call(table=None) == call(hq=7) == B.MQ_ERR_INVALID_ARG
    assert call(leader=None) == call(shared=None) == call(q=None) == call(o=None) == call(ws=None) == B.MQ_ERR_INVALID_ARG
    assert call(n_seq=1025) == call(total=1 << 28, max_q=1, hq=8) == call(cache=_cache(dim=96)) == B.MQ_ERR_UNSUPPORTED
    for bad in (0.0, -1.0, float("nan"), float("inf")):
        assert call(scale=bad) == B.MQ_ERR_INVALID_ARG
    assert call(ldq=1016) == call(ldo=512) == B.MQ_ERR_INVALID_ARG
    assert call(q=A + 2) == call(o=A + 8) == call(ldq=1028) == call(ws=A + 16) == B.MQ_ERR_ALIGNMENT
    size = lambda n=2, total=5, max_q=4: lib.mq_kv_attention_shared_workspace_bytes(C.byref(B.mq_kv_batch(n, total, max_q, 7, A, A, A, None)), C.byref(_cache()), 8)
    assert size() > 2 * 5 * 8 * 128 * 4 and call(wsb=size() - 1) == B.MQ_ERR_WORKSPACE
    assert size(n=1025) == size(max_q=6) == 0
    assert call(n_seq=0, total=0, max_q=0) == call(total=0, max_q=0) == B.MQ_OK     # nothing to do


# ------------------------------------------------------------------------------------------------ the cache whose bookkeeping is on the GPU
class _State:
    def __init__(self, kv_len, seen, table, free, n_free, page, borrowed=None):
        self.t = dict(kv_len=kv_len, seen=seen, table=table, free=free, n_free=n_free, borrowed=borrowed)
        self.page = page


def _plan(state, new, cu, slots, pos, status=None, keep=None):
    """mq_kv_plan on the CPU, by the oracle."""
    t = state.t
    host = {k: t[k].tolist() for k in ("kv_len", "seen", "borrowed", "table")}
    host.update(free=t["free"][:int(t["n_free"])].tolist(), n_pages=len(t["free"]))
    try:
        got = P.plan(host, new.tolist(), None if keep is None else keep.tolist(), len(slots), state.page)
    except P.Refused as e:
        cu.zero_(), slots.fill_(-1), pos.zero_()
        status[:] = torch.tensor([B.MQ_ERR_WORKSPACE, e.args[0]])
        return
    for to, v in zip((cu, slots, pos), got):
        to[:] = torch.tensor(v, dtype=to.dtype)
    for k in ("kv_len", "seen", "borrowed", "table"):
        t[k][:] = torch.tensor(host[k], dtype=torch.int32)
    t["free"][:len(host["free"])] = torch.tensor(host["free"], dtype=torch.int32)
    t["n_free"][0] = len(host["free"])


class _Handle:
    def __init__(self, K, V, k_scale=None, v_scale=None):
        self.n_kv_heads, self.head_dim, self.page_size, self.device = K.shape[1], K.shape[3], K.shape[2], K.device


@pytest.fixture
def make(monkeypatch):
    monkeypatch.setattr(B, "KVCache", _Handle)
    monkeypatch.setattr(B, "KVState", _State)
    monkeypatch.setattr(B, "mq_kv_plan", _plan)
    monkeypatch.setattr(B, "mq_last_device_status", lambda ws: (int(ws[0]), 0))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    return lambda *args, **kw: KC.DeviceKVCache(*args, device="cpu", **kw)


def _pages(cache, b):
    return cache.table[b, :-(-int(cache.kv_len[b]) // cache.page_size)].tolist()


def test_steps_of_the_device_cache_and_their_undoing(make):
    cache = make(3, 12, 100, 2, 64, page_size=16)
    step = cache.extend([20, 0, 33])
    assert step.cu_q.tolist() == [0, 20, 20, 53] and step.total == 53 and step.max_q == 33 and step.cu_q_host(2) == 20
    assert cache.lengths() == [20, 0, 33] and int(cache.n_free) == 7 and step.pos.tolist() == list(range(20)) + list(range(33))
    free = cache.free[:7].tolist()
    again = cache.extend([1, 40, 1])
    cache.undo(again)
    assert cache.lengths() == [20, 0, 33] and cache.free[:int(cache.n_free)].tolist() == free and cache.seen.tolist() == [20, 0, 33]
    for s in (step, again):
        with pytest.raises(RuntimeError):
            cache.undo(s)
    assert cache.status_ok()
    refused = cache.extend([93, 0, 0])                       # behind the seven pages of max_len: no rows, nothing changes
    assert refused.cu_q.tolist() == [0] * 4 and set(refused.slots.tolist()) == {-1} and cache.lengths() == [20, 0, 33]
    cache.undo(refused)
    assert cache.lengths() == [20, 0, 33] and not cache.status_ok()
    cache.extend([5, 1, 1], keep=[10, 9, 0])
    assert cache.lengths() == [15, 1, 1] and cache.seen.tolist() == [15, 1, 1]


def test_sharing_in_the_device_cache(make):
    cache = make(6, 40, 200, 2, 64, page_size=16)
    cache.extend([70, 0, 0, 0, 30, 0])
    assert cache.share(0, 1, 2) == 64
    assert cache.lengths() == [70, 64, 64, 0, 30, 0] and cache.seen.tolist() == [70, 64, 64, 0, 30, 0]
    assert _pages(cache, 1) == _pages(cache, 0)[:4] and cache.leaders == [0, 0, 0, 3, 4, 5] == cache.leader.tolist()
    assert cache.share(0, 3, 1) == 64
    for src, first, count in ((1, 4, 1), (4, 3, 1), (0, 5, 1), (4, 5, 2), (4, 5, 0), (0, 4, 1)):
        with pytest.raises(RuntimeError):
            cache.share(src, first, count)
    before = int(cache.n_free)
    cache.extend([1, 6, 7, 20, 0, 0])
    assert cache.lengths() == [71, 70, 71, 84, 30, 0] and before - int(cache.n_free) == 4
    assert all(_pages(cache, b)[4:] and not set(_pages(cache, b)[4:]) & set(_pages(cache, 0)) for b in (1, 2, 3))
    most = 1 << 30
    for call in (lambda: cache.release([0]), lambda: cache.release([0, 1]), lambda: cache.extend([0] * 6, keep=[60] + [most] * 5),
                 lambda: cache.extend([0] * 6, keep=[most, 0] + [most] * 4), lambda: cache.extend([0] * 6, keep=[most, 48] + [most] * 4),
                 lambda: cache.release([-1]), lambda: cache.release([6])):
        with pytest.raises(RuntimeError):
            call()
    cache.release([1, 3])
    assert cache.lengths() == [71, 0, 71, 0, 30, 0] and cache.leaders == [0, 1, 0, 3, 4, 5] and cache.borrowed.tolist() == [0, 0, 4, 0, 0, 0]
    cache.release([0, 2])
    assert int(cache.n_free) == 40 - 2 and cache.leader.tolist() == list(range(6)) and cache.leaders == list(range(6))
    cache.extend([0] * 6, keep=[0] * 6)
    assert int(cache.n_free) == 40 and sorted(cache.free.tolist()) == list(range(40)) and cache.status_ok()


def test_numbers_of_the_device_cache_stay_few(make):
    cache = make(2, 1000, 4000, 2, 64, page_size=16)
    for n in range(600):
        cache.extend([n % 300, 0], keep=[n % 7, n])
    assert len(cache._numbers) <= 256


def test_the_shared_form_is_called_where_it_saves_enough(make):
    cache = make(6, 40, 200, 2, 64, page_size=16)        # 256 numbers to a key
    cache.extend([70, 0, 0, 40, 0, 0])
    cache.share(0, 1, 2)
    cache.share(3, 4, 2)
    step = cache.extend([1] * 6)
    for new, numbers in (([1] * 6, (2 * 64 + 2 * 32) * 256), ([0, 1, 1, 0, 0, 0], 64 * 256), ([1, 0, 1, 1, 0, 0], 64 * 256), ([0, 1, 0, 1, 0, 0], None),
                         ([1, 0, 0, 1, 0, 0], None)):
        step.new = new
        for limit, shared in ((0, True), (numbers or 0, True), ((numbers or 0) + 1, False)):
            cache.shared_from = limit
            assert cache._shares(step) == (shared and numbers is not None)
    cache.shared_from = 0
    cache.release([1, 2, 4, 5])
    assert not cache._shares(cache.extend([1] * 6))
    wide = make(1025, 1100, 32, 1, 64, page_size=16, shared_from=0)
    wide.extend([20] + [0] * 1024)
    wide.share(0, 1, 2)
    assert not wide._shares(wide.extend([1] * 1025))


def test_an_answer_that_ends_leaves_the_others_their_sharing(make):
    cache = make(8, 80, 200, 2, 64, page_size=16, shared_from=0)
    cache.extend([70] + [0] * 6 + [5])
    cache.share(0, 1, 6)
    step = cache.extend([1] * 8)
    cache.release([2])                                        # nobody parts the group as long as the place is empty
    assert cache.leader.tolist() == [0, 0, 0, 0, 0, 0, 0, 7] and cache.leaders == [0, 0, 2, 0, 0, 0, 0, 7]
    step = cache.extend([1, 1, 0, 1, 1, 1, 1, 1])
    saved = lambda step: [limit for limit in (5, 4, 3, 2, 1) if not setattr(cache, "shared_from", limit * 64 * 256) and cache._shares(step)]
    assert saved(step)[0] == 5                                # (64 keys of 256 numbers for five of six)
    cache.release([4, 6])
    assert cache.leader.tolist() == [0, 0, 0, 0, 0, 0, 6, 7]
    step = cache.extend([1, 0, 9, 1, 0, 1, 0, 0])             # place 2 taken by a sequence of its own: two groups, read by what both sides' pages are
    assert cache.leader.tolist() == [0, 0, 2, 3, 3, 3, 6, 7] and cache.lengths()[:6] == [73, 66, 9, 67, 0, 67]
    assert cache.shared_len.tolist()[3:6] == [64, 0, 64] and _pages(cache, 3)[:4] == _pages(cache, 0)[:4] == _pages(cache, 5)[:4]
    assert saved(step) == [1] and saved(cache.extend([1, 1, 1, 1, 0, 1, 0, 0]))[0] == 2
    assert saved(cache.extend([1, 0, 1, 0, 0, 1, 0, 0])) == []                               # one of each group: nothing is read twice
    assert saved(cache.extend([0] * 8)) == []
    cache.release([2])
    assert cache.leader.tolist() == [0, 0, 0, 0, 0, 0, 6, 7]
    cache.release([0, 1, 3, 5])
    assert cache.leader.tolist() == list(range(8)) and cache.lengths() == [0] * 7 + [7] and cache.status_ok()
    assert not cache._shares(cache.extend([1] * 8))
    assert not any(cache._ended)
    cache.extend([0] * 8, keep=[0] * 8)
    assert int(cache.n_free) == 80


def test_groups_do_not_change_in_a_capture(make, monkeypatch):
    cache = make(4, 40, 200, 2, 64, page_size=16)
    cache.extend([40, 0, 0, 0])
    cache.share(0, 1, 3)
    cache.extend([0, 1, 1, 1])
    cache.release([2])
    for row in ([1, 1, 3, 1], [0, 0, 2, 3], [0, 0, 0, 0]):          # (the arrays are there)
        cache._ints(row)
    with monkeypatch.context() as m:
        m.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
        with pytest.raises(RuntimeError, match="once before"):
            cache.extend([1, 1, 3, 1])
        assert cache.leader.tolist() == [0, 0, 0, 0] == cache._heads and cache.lengths() == [40, 33, 0, 33]
    cache.extend([1, 1, 3, 1])
    assert cache.leader.tolist() == [0, 0, 2, 3] == cache._heads
    with monkeypatch.context() as m:
        m.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
        cache.extend([1, 1, 3, 1])
    assert cache.lengths() == [42, 35, 6, 35] and cache.status_ok()
