"""Host-side checks of the key/value-cache entry points (no GPU): refusals before anything is enqueued, workspace sizes,
and pins of the float64 oracle."""
import ctypes as C
import os

import numpy as np
import pytest

from oracle import kv_oracle as O
from paper_2502_00425_b200 import binding as B
from paper_2502_00425_b200 import build

A = 0x10000   # a fake, aligned device address: validation must come before it is used


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return B.load()


def _cache(K=A, V=A, page_stride=4 * 64 * 128, head_stride=64 * 128, slot_stride=128, n_pages=10, page=64, hkv=4, dim=128, flags=0,
           ks=None, vs=None):
    return B.mq_kv_cache(K, V, page_stride, head_stride, slot_stride, n_pages, page, hkv, dim, flags, ks, vs)


def _batch(n_seq=2, total=5, max_q=4, max_pages=7, cu=A, kv=A, table=A, perm=None):
    return B.mq_kv_batch(n_seq, total, max_q, max_pages, cu, kv, table, perm)


BAD_CACHES = [
    (dict(flags=2), "MQ_ERR_INVALID_ARG"),
    (dict(dim=96), "MQ_ERR_UNSUPPORTED"),
    (dict(page=48), "MQ_ERR_UNSUPPORTED"),
    (dict(page=8), "MQ_ERR_UNSUPPORTED"),
    (dict(page=512), "MQ_ERR_UNSUPPORTED"),
    (dict(page=0), "MQ_ERR_INVALID_ARG"),
    (dict(n_pages=-1), "MQ_ERR_INVALID_ARG"),
    (dict(hkv=0), "MQ_ERR_INVALID_ARG"),
    (dict(K=None), "MQ_ERR_INVALID_ARG"),
    (dict(slot_stride=64), "MQ_ERR_INVALID_ARG"),           # rows would overlap
    (dict(head_stride=-128), "MQ_ERR_INVALID_ARG"),
    (dict(V=A + 8), "MQ_ERR_ALIGNMENT"),
    (dict(slot_stride=132), "MQ_ERR_ALIGNMENT"),
    (dict(page_stride=1 << 40), "MQ_ERR_UNSUPPORTED"),
    (dict(flags=1), "MQ_ERR_INVALID_ARG"),                  # int8 without scales
    (dict(ks=A, vs=A), "MQ_ERR_INVALID_ARG"),               # scales without int8
    (dict(flags=1, ks=A, vs=A, slot_stride=136), "MQ_ERR_ALIGNMENT"),
]


@pytest.mark.parametrize("kw,status", BAD_CACHES)
def test_every_entry_point_refuses_a_bad_cache(lib, kw, status):
    c, good = _cache(**kw), _cache()
    want = getattr(B, status)
    b = _batch()
    att = lib.mq_kv_attention(A, 1024, C.byref(b), C.byref(c), 8, 0.1, A, 1024, None, A, 1 << 30, None)
    assert att == want and lib.mq_kv_attention_workspace_bytes(C.byref(b), C.byref(c), 8) == 0
    assert lib.mq_kv_weights(A, 1024, C.byref(b), C.byref(c), 8, 0.1, A, None, A, 4096, 512, 448, None, None) == want
    for src, dst in ((c, good), (good, c)):
        assert lib.mq_kv_evict(C.byref(src), A, 7, A, 2, A, 4096, 512, 448, 64, 0, 0, C.byref(dst), A, 7, A, A, None, None) == want
    if kw.get("dim", 128) == 128 and kw.get("hkv", 4) == 4:
        assert lib.mq_qk_norm_rope(A, 1024, A, 512, A, 512, 5, 8, 4, 128, None, None, 1e-6, A, 1e4, 0, A, 1024, None, 0,
                                   C.byref(c), A, None) == want


def test_attention_refusals(lib):
    def call(q=A, ldq=1024, hq=8, scale=0.1, o=A, ldo=1024, ws=A, wsb=1 << 30, cache=None, **kw):
        return lib.mq_kv_attention(q, ldq, C.byref(_batch(**kw)), C.byref(cache or _cache()), hq, scale, o, ldo, None, ws, wsb, None)

    assert lib.mq_kv_attention(A, 1024, None, C.byref(_cache()), 8, 0.1, A, 1024, None, A, 1 << 30, None) == B.MQ_ERR_INVALID_ARG
    assert lib.mq_kv_attention(A, 1024, C.byref(_batch()), None, 8, 0.1, A, 1024, None, A, 1 << 30, None) == B.MQ_ERR_INVALID_ARG
    assert call(n_seq=-1) == call(total=-1) == call(max_q=-1) == call(max_pages=-1) == B.MQ_ERR_INVALID_ARG
    assert call(max_q=6) == B.MQ_ERR_INVALID_ARG                     # more rows in one sequence than in all
    assert call(n_seq=5000) == B.MQ_ERR_UNSUPPORTED
    assert call(max_pages=1 << 23) == B.MQ_ERR_UNSUPPORTED
    assert call(cu=None) == call(kv=None) == call(table=None) == B.MQ_ERR_INVALID_ARG
    assert call(hq=7) == call(hq=0) == B.MQ_ERR_INVALID_ARG
    for bad in (0.0, -1.0, float("nan"), float("inf")):
        assert call(scale=bad) == B.MQ_ERR_INVALID_ARG
    assert call(ldq=1016) == call(ldo=512) == B.MQ_ERR_INVALID_ARG
    assert call(q=None) == call(o=None) == call(ws=None) == B.MQ_ERR_INVALID_ARG
    assert call(q=A + 2) == call(o=A + 8) == call(ldq=1028) == call(ldo=1026) == call(ws=A + 16) == B.MQ_ERR_ALIGNMENT
    assert call(wsb=256) == B.MQ_ERR_WORKSPACE
    need = lib.mq_kv_attention_workspace_bytes(C.byref(_batch()), C.byref(_cache()), 8)
    assert need > 256 and call(wsb=need - 1) == B.MQ_ERR_WORKSPACE
    assert call(n_seq=0, total=0, max_q=0) == call(total=0, max_q=0) == B.MQ_OK     # nothing to do


def test_weights_refusals(lib):
    def call(q=A, ldq=1024, hq=8, scale=0.1, lse=A, w=A, ss=4096, hs=512, wk=448, **kw):
        return lib.mq_kv_weights(q, ldq, C.byref(_batch(**kw)), C.byref(_cache()), hq, scale, lse, None, w, ss, hs, wk, None, None)

    assert call(hq=6) == call(ldq=512) == call(scale=0.0) == call(ss=-1) == call(hs=-1) == call(wk=-1) == B.MQ_ERR_INVALID_ARG
    assert call(q=None) == call(lse=None) == call(w=None) == B.MQ_ERR_INVALID_ARG
    assert call(q=A + 2) == call(ldq=1028) == B.MQ_ERR_ALIGNMENT
    assert call(n_seq=0, total=0, max_q=0) == call(max_pages=0) == call(wk=0) == B.MQ_OK


def test_weights_refuse_rows_that_share_entries(lib):
    def call(ss, hs, wk, max_pages=7):      # two sequences of four heads, 7 pages of 64 keys
        return lib.mq_kv_weights(A, 1024, C.byref(_batch(max_pages=max_pages)), C.byref(_cache()), 8, 0.1, A, None, A, ss, hs, wk, None, None)

    assert call(0, 448, 448) == call(4 * 448, 0, 448) == call(0, 0, 448) == B.MQ_ERR_INVALID_ARG     # (expanded tensors)
    assert call(4 * 448, 447, 448) == call(4 * 448 - 1, 448, 448) == call(448, 2 * 448 - 1, 448) == B.MQ_ERR_INVALID_ARG
    assert call(4 * 128, 128, 448, max_pages=0) == B.MQ_OK                                           # (nothing to do)


def test_evict_refusals(lib):
    def call(src=None, dst=None, table=A, mp=7, kv=A, n=2, w=A, ss=4096, hs=512, wk=448, budget=64, first=0, last=0, dt=A, dmp=7, kept=A, nl=A):
        return lib.mq_kv_evict(C.byref(src or _cache()), table, mp, kv, n, w, ss, hs, wk, budget, first, last, C.byref(dst or _cache()), dt,
                               dmp, kept, nl, None, None)

    assert call(dst=_cache(hkv=2)) == call(dst=_cache(dim=64)) == B.MQ_ERR_INVALID_ARG
    assert call(dst=_cache(flags=1, ks=A, vs=A)) == B.MQ_ERR_INVALID_ARG           # another type
    assert call(budget=-1) == call(first=-1) == call(last=-1) == call(n=-1) == call(mp=-1) == call(wk=-1) == B.MQ_ERR_INVALID_ARG
    assert call(first=33, last=32) == B.MQ_ERR_INVALID_ARG                          # more than the budget
    assert call(budget=449) == B.MQ_ERR_INVALID_ARG                                 # 7 pages of 64 hold 448
    assert call(n=5000) == B.MQ_ERR_UNSUPPORTED
    assert call(table=None) == call(kv=None) == call(w=None) == call(dt=None) == call(kept=None) == call(nl=None) == B.MQ_ERR_INVALID_ARG
    assert call(n=0) == B.MQ_OK


def test_evict_refuses_outputs_over_its_inputs(lib):
    """Refused before anything is enqueued (an accepted call would go to a device)."""
    def call(kv=A, w=0x1000000, nl=A, w_out=None):
        return lib.mq_kv_evict(C.byref(_cache()), A, 7, kv, 2, w, 4096, 512, 448, 64, 0, 0, C.byref(_cache()), A, 7, A, nl, w_out, None)

    assert call(nl=A + 4) == call(nl=A - 4) == B.MQ_ERR_INVALID_ARG                 # lengths that overlap in part
    # kept weights in the memory of the weights: W ends (2 - 1) * 4096 + 3 * 512 + 448 elements behind its start, W_out 2 * 4 * 64
    w, w_end, o_len = 0x1000000, (4096 + 3 * 512 + 448) * 4, 2 * 4 * 64 * 4
    assert call(w_out=w) == call(w_out=w + w_end - 4) == call(w_out=w - o_len + 4) == B.MQ_ERR_INVALID_ARG


def test_norm_rope_refusals(lib):
    def call(q=A, ldq=1024, k=A, ldk=512, v=A, ldv=512, T=5, hq=8, hkv=4, dim=128, gq=None, gk=None, eps=1e-6, pos=A, base=1e4, flags=0,
             qo=A, ldqo=1024, ko=None, ldko=0, cache=None, slots=A, none=False):
        c = None if none else C.byref(cache or _cache())
        return lib.mq_qk_norm_rope(q, ldq, k, ldk, v, ldv, T, hq, hkv, dim, gq, gk, eps, pos, base, flags, qo, ldqo, ko, ldko, c, slots, None)

    assert call(T=-1) == call(hq=0) == call(hkv=0) == call(flags=2) == call(eps=-1.0) == call(base=1.0) == B.MQ_ERR_INVALID_ARG
    assert call(eps=float("nan")) == call(base=float("inf")) == B.MQ_ERR_INVALID_ARG
    assert call(dim=32, none=True, ko=A, ldko=512) == B.MQ_ERR_UNSUPPORTED
    assert call(cache=_cache(hkv=2)) == call(cache=_cache(dim=64)) == B.MQ_ERR_INVALID_ARG
    assert call(ldq=1000) == call(ldk=256) == call(ldv=256) == call(ldqo=512) == call(ko=A, ldko=256) == B.MQ_ERR_INVALID_ARG
    assert call(q=None) == call(k=None) == call(v=None) == call(pos=None) == call(slots=None) == call(qo=None) == B.MQ_ERR_INVALID_ARG
    assert call(none=True) == B.MQ_ERR_INVALID_ARG                                  # neither a cache nor K_out
    assert call(q=A + 2) == call(ldk=516) == call(gq=A + 4) == call(ko=A + 2, ldko=512) == call(ldqo=1028) == B.MQ_ERR_ALIGNMENT
    assert call(T=0) == B.MQ_OK


def test_binding_refuses_mismatched_tensors():
    import torch
    K = torch.zeros((2, 2, 16, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        B.KVCache(K, K.transpose(1, 2).contiguous().transpose(1, 2))                # other strides
    with pytest.raises(ValueError):
        B.KVCache(K, K, torch.ones(2), torch.ones(2))                               # scales on a bf16 cache
    with pytest.raises(ValueError):
        B.KVCache(K.to(torch.int8), K.to(torch.int8))                               # an int8 cache without scales
    with pytest.raises(ValueError):
        B.KVCache(K, K.clone())                                                     # host memory


@pytest.mark.parametrize("kw", [
    dict(page_stride=128, head_stride=128, slot_stride=128),                                # all rows in one place
    dict(page_stride=4 * 64 * 128, head_stride=128, slot_stride=256),                       # four heads in room for two
    dict(page_stride=4 * 64 * 128 - 128, head_stride=64 * 128, slot_stride=128),            # a page's end over the next one's start
    dict(page_stride=128, head_stride=10 * 128, slot_stride=40 * 128 - 64),
])
def test_writers_refuse_a_cache_whose_rows_overlap(lib, kw):
    c, good = _cache(**kw), _cache()
    assert lib.mq_qk_norm_rope(A, 1024, A, 512, A, 512, 5, 8, 4, 128, None, None, 1e-6, A, 1e4, 0, A, 1024, None, 0,
                               C.byref(c), A, None) == B.MQ_ERR_INVALID_ARG
    assert lib.mq_kv_evict(C.byref(good), A, 7, A, 2, A, 4096, 512, 448, 64, 0, 0, C.byref(c), A, 7, A, A, None, None) == B.MQ_ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [
    dict(page_stride=128, head_stride=10 * 128, slot_stride=40 * 128),                      # any order of the dimensions
    dict(page_stride=64 * 160, head_stride=1 << 30, slot_stride=160),
    dict(page_stride=128, n_pages=1),                                                       # a stride that is never taken
])
def test_writers_take_rows_in_any_order(lib, kw):
    assert lib.mq_qk_norm_rope(A, 1024, A, 512, A, 512, 0, 8, 4, 128, None, None, 1e-6, A, 1e4, 0, A, 1024, None, 0,
                               C.byref(_cache(**kw)), A, None) == B.MQ_OK                   # no rows: nothing is enqueued
    assert lib.mq_kv_evict(C.byref(_cache()), A, 7, A, 0, A, 4096, 512, 448, 64, 0, 0, C.byref(_cache(**kw)), A, 7, A, A, None, None) == B.MQ_OK


def test_roles_of_the_cache_kernels_meet_at_bounded_waits_only():
    """A barrier over some of a CTA's warps (bar.sync / bar.red with a name) has no limit: a warp that gave up on a bounded wait
    would leave the others at it for good.  The roles of these kernels are ordered by mbarriers, whose waits expire."""
    src = os.path.join(os.path.dirname(build.__file__), "csrc")
    names = [f for f in os.listdir(src) if f.startswith("mq_kv")]
    assert "mq_kv_weights_chunk.cu" in names and "mq_kv_chunk.cu" in names
    for f in names:
        text = open(os.path.join(src, f)).read()
        assert "named_bar" not in text and "bar.sync" not in text and "bar.red" not in text, f


# ------------------------------------------------------------------------------------------------ the oracle
def test_oracle_visibility_reduces_to_the_dense_masks():
    from oracle import mq_oracle as M
    rng = np.random.default_rng(0)
    vis = rng.random(23) < 0.5
    perm = np.concatenate([np.flatnonzero(vis), np.flatnonzero(~vis)])
    see = O.visible(23, 40, perm)
    assert see[:, :17].all()
    assert np.array_equal(see[:, 17:], perm[None, :] <= perm[:, None])
    assert np.array_equal(O.visible(5, 5), np.tril(np.ones((5, 5), bool)))
    assert np.array_equal(O.visible(3, 2), [[False, False], [True, False], [True, True]])   # the first row sees nothing
    x = rng.standard_normal((7, 16))
    assert np.allclose(O.norm_rope(x[:, None], None, 1e-6, np.arange(7) * 100, 10000.0, False)[0][:, 0],
                       M.rope(x.astype(np.float32), np.arange(7) * 100), atol=1e-6)


def test_oracle_softmax_weights_and_eviction_pins():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((4, 8)), rng.standard_normal((9, 8)), rng.standard_normal((9, 8))
    o, lse, p, _, _ = O.attention(q, k, v, 0.5)
    assert np.allclose(p.sum(1), 1) and np.allclose(o, p @ v)
    assert np.allclose(O.weights([q], k, [lse], 0.5), p.sum(0))
    assert O.keep(np.array([5.0, 1, 4, 4, 9, 0]), 6, 4, 1, 1).tolist() == [0, 2, 4, 5]
    assert O.keep(np.array([0.0, 2, 2, 2, 0]), 5, 3, 0, 1).tolist() == [1, 2, 4]             # ties: the lowest index
    assert O.keep(np.array([np.nan, -np.inf, 1.0]), 3, 2, 0, 0).tolist() == [1, 2]
    y, _ = O.norm_rope(np.ones((1, 1, 4)) * 3, np.array([1.0, 2, 3, 4]), 0.0, [0], 10000.0, True)
    assert np.allclose(y, [[[1, 2, 3, 4]]])
