"""mq_qk_norm_rope (norm, rotary embedding, store into the paged cache) against the float64 definition.

Tolerance: half a bf16 step of the result, 2^-8 |y|, plus the float32 arithmetic in front of it (sum of squares, rsqrt,
gain, sine and cosine, two products): fewer than 32 roundings of 2^-24, relative to the magnitudes of the pair's two
normed channels.  An int8 code is the value over the scale, off by half a step and the same arithmetic.
"""
import numpy as np
import pytest
import torch

from oracle import kv_oracle as O
from paper_2502_00425_b200 import binding as B

from kv_util import DEV

pytestmark = pytest.mark.gpu


def _pool(n_pages, hkv, page, dim, int8, layout):
    dt = torch.int8 if int8 else torch.bfloat16
    fill = 99
    if layout == "token":
        return [torch.full((n_pages, page, hkv, dim), fill, dtype=dt, device=DEV).permute(0, 2, 1, 3) for _ in range(2)]
    return [torch.full((n_pages, hkv, page, dim), fill, dtype=dt, device=DEV) for _ in range(2)]


def _close(got, ref, mag):
    return np.all(np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -19 * mag + 1e-38)


@pytest.mark.parametrize("T,hq,hkv,dim,half,norm,int8,layout,far", [
    (1, 28, 4, 128, False, "qk", False, "head", 0),
    (5, 4, 2, 64, True, "qk", False, "token", 0),
    (33, 32, 8, 128, True, "", False, "token", 30000),
    (33, 3, 3, 64, False, "q", True, "head", 30000),
    (7, 28, 4, 128, False, "k", True, "token", 1 << 22),
    (1200, 28, 4, 128, False, "qk", False, "head", 0),      # many rows: the variant with several loads in flight
    (1500, 12, 4, 64, True, "qk", True, "head", 100000),
    (2300, 5, 1, 128, True, "qk", False, "head", 1000),
])
def test_norm_rope_append(T, hq, hkv, dim, half, norm, int8, layout, far):
    rng = np.random.default_rng(T + dim)
    page, n_pages = 16, T // 16 + 4
    width = (hq + 2 * hkv) * dim
    # q, k, v as column ranges of one stacked projection, its pitch wider than its columns
    qkv = torch.from_numpy((rng.standard_normal((T, width + 8)) * 3).astype(np.float32)).to(torch.bfloat16)
    qkv[0, :dim] = 0.0
    dq = qkv.to(DEV)
    q, k, v = dq[:, :hq * dim], dq[:, hq * dim:(hq + hkv) * dim], dq[:, (hq + hkv) * dim:width]
    pos = (rng.permutation(T) + far).astype(np.int32)
    gains = {c: (1 + 0.2 * rng.standard_normal(dim)).astype(np.float32) if c in norm else None for c in "qk"}
    dg = {c: None if g is None else torch.from_numpy(g).to(DEV) for c, g in gains.items()}
    K, V = _pool(n_pages, hkv, page, dim, int8, layout)
    scales = [torch.from_numpy((0.02 + 0.02 * rng.random(hkv)).astype(np.float32)) for _ in range(2)] if int8 else [None, None]
    cache = B.KVCache(K, V, *(None if s is None else s.to(DEV) for s in scales))
    slots = rng.permutation(n_pages * page)[:T].astype(np.int64)
    if T > 4:
        slots[2], slots[4] = -1, n_pages * page        # padding, and a slot behind the cache: not stored
    q_out = torch.full((T + 1, hq * dim), 5.0, dtype=torch.bfloat16, device=DEV)
    k_out = torch.full((T + 1, hkv * dim), 5.0, dtype=torch.bfloat16, device=DEV)
    B.mq_qk_norm_rope(q, k, torch.from_numpy(pos).to(DEV), hq, hkv, q_out[:T], k_out=k_out[:T], gain_q=dg["q"], gain_k=dg["k"],
                      base=10000.0, half=half, v=v, cache=cache, slots=torch.from_numpy(slots).to(DEV))
    torch.cuda.synchronize()
    host = qkv.double().numpy()
    yq, mq_ = O.norm_rope(host[:, :hq * dim].reshape(T, hq, dim), gains["q"], 1e-6, pos, 10000.0, half)
    yk, mk = O.norm_rope(host[:, hq * dim:(hq + hkv) * dim].reshape(T, hkv, dim), gains["k"], 1e-6, pos, 10000.0, half)
    back = lambda t: t.double().cpu().numpy()
    assert _close(back(q_out[:T]).reshape(T, hq, dim), yq, mq_)
    assert _close(back(k_out[:T]).reshape(T, hkv, dim), yk, mk)
    assert bool((q_out[T:] == 5.0).all()) and bool((k_out[T:] == 5.0).all())
    vals = host[:, (hq + hkv) * dim:width].reshape(T, hkv, dim)
    ok = (slots >= 0) & (slots < n_pages * page)
    flat = lambda c: back(c.permute(0, 2, 1, 3).reshape(-1, hkv, dim))
    fk, fv = flat(K), flat(V)
    if not int8:
        assert np.array_equal(fk[slots[ok]], back(k_out[:T]).reshape(T, hkv, dim)[ok])   # one rounding, the same one
        assert np.array_equal(fv[slots[ok]], vals[ok])
    else:
        for got, y, mag, s in ((fk, yk, mk, scales[0]), (fv, vals, np.abs(vals), scales[1])):
            want, unit = y / s.double().numpy()[:, None], s.double().numpy()[:, None]
            lim = np.clip(want, -128, 127)
            assert np.all(np.abs(got[slots[ok]] - lim[ok]) <= 0.5 + (2.0 ** -19 * mag / unit + 2.0 ** -22 * np.abs(want))[ok])
    rest = np.setdiff1d(np.arange(n_pages * page), slots[ok])
    assert np.all(fk[rest] == 99) and np.all(fv[rest] == 99)                            # nothing else was touched


def test_in_place_and_without_a_cache_equals_the_stored_form():
    rng = np.random.default_rng(5)
    T, hq, hkv, dim = 19, 6, 2, 128
    q = torch.from_numpy(rng.standard_normal((T, hq * dim)).astype(np.float32)).to(torch.bfloat16).to(DEV)
    k = torch.from_numpy(rng.standard_normal((T, hkv * dim)).astype(np.float32)).to(torch.bfloat16).to(DEV)
    pos = torch.arange(T, dtype=torch.int32, device=DEV) * 17
    gain = torch.ones(dim, device=DEV)
    for half in (False, True):
        qo, ko = torch.empty_like(q), torch.empty_like(k)
        B.mq_qk_norm_rope(q, k, pos, hq, hkv, qo, k_out=ko, gain_q=gain, gain_k=gain, half=half)
        q2, k2 = q.clone(), k.clone()
        K, V = _pool(2, hkv, 16, dim, False, "head")
        B.mq_qk_norm_rope(q2, k2, pos, hq, hkv, q2, k_out=k2, gain_q=gain, gain_k=gain, half=half, v=k, cache=B.KVCache(K, V),
                          slots=torch.arange(T, dtype=torch.int64, device=DEV))
        assert torch.equal(q2, qo) and torch.equal(k2, ko)
        assert torch.equal(K.permute(0, 2, 1, 3).reshape(-1, hkv * dim)[:T], ko)
        assert torch.equal(V.permute(0, 2, 1, 3).reshape(-1, hkv * dim)[:T], k)


def test_pair_rotation_agrees_with_the_rope_glue_kernel():
    """Without gains this is mq_glue_rope's rotation (up to that kernel's float32 angle)."""
    rng = np.random.default_rng(6)
    T, hq, dim = 40, 4, 128
    q = torch.from_numpy(rng.standard_normal((T, hq * dim)).astype(np.float32)).to(torch.bfloat16).to(DEV)
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    a, b, kk = torch.empty_like(q), torch.empty_like(q), torch.empty_like(q)
    B.mq_qk_norm_rope(q, q, pos, hq, hq, a, k_out=kk)
    B.mq_glue_rope(q, pos, hq, b)
    assert torch.equal(a, kk)
    d = (a.float() - b.float()).abs()
    assert bool((d <= 2.0 ** -7 * b.float().abs() + 1e-4).all())   # one bf16 step at most, and 40 * 2^-23 rad of angle


def test_far_offsets_of_a_large_pool():
    """A page stride that puts the last pages behind 2^32 bytes: byte offsets are 64-bit."""
    hkv, dim, page = 2, 128, 16
    stride = 1 << 20                                   # elements between pages: 2 MiB
    n_pages = 2100                                     # the last page starts behind 4.4e9 bytes
    pool = torch.empty((n_pages - 1) * stride + hkv * page * dim, dtype=torch.bfloat16, device=DEV)
    K = pool.as_strided((n_pages, hkv, page, dim), (stride, page * dim, dim, 1))
    V = pool.as_strided((n_pages, hkv, page, dim), (stride, page * dim, dim, 1), storage_offset=0)
    for p in (0, n_pages - 1):
        K[p] = 0
    cache = B.KVCache(K, K.as_strided(K.shape, K.stride(), 0))
    x = torch.randn((2, hkv * dim), device=DEV).to(torch.bfloat16)
    pos = torch.zeros(2, dtype=torch.int32, device=DEV)
    out = torch.empty_like(x)
    slots = torch.tensor([3, (n_pages - 1) * page + 5], dtype=torch.int64, device=DEV)
    B.mq_qk_norm_rope(x, x, pos, hkv, hkv, out, v=x, cache=cache, slots=slots)   # position 0: the rotation is the identity
    torch.cuda.synchronize()
    assert torch.equal(V[0, :, 3].reshape(-1), x[0]) and torch.equal(V[n_pages - 1, :, 5].reshape(-1), x[1])
    # and the attention reads them from there
    ws = B.new_kv_attention_workspace(1, 1, 1, 1, hkv, cache)
    table = torch.tensor([[n_pages - 1]], dtype=torch.int32, device=DEV)
    one = torch.tensor([6], dtype=torch.int32, device=DEV)
    K[n_pages - 1, :, :5] = -x[1].view(hkv, 1, dim) * 100        # keys that lose against slot 5
    o = torch.empty((1, hkv * dim), dtype=torch.bfloat16, device=DEV)
    B.mq_kv_attention(x[1:] * 30, torch.tensor([0, 1], dtype=torch.int32, device=DEV), one, table, cache, hkv, 1, o, ws)
    assert torch.equal(o[0], x[1])


@pytest.mark.parametrize("int8", [False, True])
def test_far_rows_of_keys_and_of_values_are_told_apart(int8):
    """K and V share one allocation at different offsets, their last pages behind 2^32 bytes, and hold different things."""
    hkv, dim, page = 2, 128, 16
    es = 1 if int8 else 2
    rows = hkv * page * dim
    stride = (1 << 21) // es                           # elements between pages: 2 MiB
    n_pages = 2100                                     # the last page starts behind 4.4e9 bytes
    dt = torch.int8 if int8 else torch.bfloat16
    pool = torch.empty((n_pages - 1) * stride + 2 * rows, dtype=dt, device=DEV)
    K, V = (pool.as_strided((n_pages, hkv, page, dim), (stride, page * dim, dim, 1), off) for off in (0, rows))
    scales = [torch.full((hkv,), s, device=DEV) for s in (0.05, 0.03)] if int8 else [None, None]
    slots = torch.tensor([3, (n_pages - 1) * page + 5, 2049 * page + 15], dtype=torch.int64, device=DEV)
    for p in (0, 2049, n_pages - 1):
        K[p], V[p] = 77, 78
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn((3, hkv * dim), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    out = torch.empty_like(k)
    B.mq_qk_norm_rope(k, k, torch.zeros(3, dtype=torch.int32, device=DEV), hkv, hkv, out, v=v, cache=B.KVCache(K, V, *scales), slots=slots)
    torch.cuda.synchronize()                           # position 0: the rotation is the identity
    for t, slot in enumerate(slots.tolist()):
        for view, x, s in ((K, k, scales[0]), (V, v, scales[1])):
            want = x[t].view(hkv, dim)
            if int8:
                inv = 1.0 / s.cpu()                    # the stored code: round_half_even(y * (1 / scale)), both in float32
                want = (want.float().cpu() * inv[:, None]).round().clamp(-128, 127).to(torch.int8).to(DEV)
            assert torch.equal(view[slot // page, :, slot % page], want)
    for view, fill in ((K, 77), (V, 78)):
        for p in (0, 2049, n_pages - 1):
            mask = torch.ones(page, dtype=torch.bool, device=DEV)
            mask[[s % page for s in slots.tolist() if s // page == p]] = False
            assert bool((view[p][:, mask] == fill).all())
