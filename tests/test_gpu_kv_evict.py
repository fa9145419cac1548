"""mq_kv_weights and mq_kv_evict against their float64 definitions.

Weights: every term is exp of a float32 argument whose error is that of its score (a float32 sum of D products, at most
(D + 8) 2^-23 of the sum of magnitudes) plus roundings of score and log-sum-exp (2^-22 of their magnitudes) and of exp2
(2^-21); the sum of n terms adds n 2^-24.  Eviction moves bytes: everything must be equal.
"""
import numpy as np
import pytest
import torch

from oracle import kv_oracle as O
from paper_2502_00425_b200 import binding as B

from kv_util import DEV, Paged, aifs_perm, cu

pytestmark = pytest.mark.gpu


def _weights_case(new, lens, hq, hkv, dim, page, int8, aifs, seed, layout="head"):
    pg = Paged(lens, hkv, dim, page, int8, layout, seed)
    rng = np.random.default_rng(seed)
    q = torch.from_numpy((rng.standard_normal((sum(new), hq * dim)) * 1.2).astype(np.float32)).to(torch.bfloat16)
    perm = aifs_perm(rng, new) if aifs else None
    qf = q.double().numpy().reshape(-1, hq, dim)
    scale, group = dim ** -0.5, hq // hkv
    lse = np.zeros((sum(new), hq), np.float32)
    mags = np.zeros((len(new), hq))
    start = 0
    for b, n in enumerate(new):
        for h in range(hq):
            _, l, _, _, mag = O.attention(qf[start:start + n, h], pg.k[b][:, h // group], pg.v[b][:, h // group], scale,
                                          None if perm is None else perm[b])
            lse[start:start + n, h] = l
            mags[b, h] = mag.max(initial=0.0)
        start += n
    return pg, q, qf, perm, lse, mags, scale, group


@pytest.mark.parametrize("case", [
    ([1], [1], 2, 1, 128, 16, False, False),
    ([1, 1, 1], [700, 128, 33], 28, 4, 128, 64, False, False),
    ([1, 0, 2], [50, 70, 300], 16, 2, 64, 16, True, False),
    ([40, 200], [300, 200], 8, 2, 128, 32, False, False),
    ([70, 9], [333, 500], 14, 2, 128, 64, True, False),
    ([130, 33], [400, 33], 12, 4, 64, 128, False, True),
    ([100], [260], 8, 2, 128, 16, True, True),
    ([300], [700], 7, 1, 128, 64, False, False),
    ([9, 140], [4, 100], 4, 2, 128, 16, False, False),     # fewer keys than rows
    ([2, 0, 1], [19, 5, 200], 130, 1, 128, 16, False, False),   # more query heads per key/value head than a row tile holds
    ([1, 2], [130, 66], 150, 1, 64, 16, True, False),
    ([1, 1, 1, 1], [64, 63, 65, 1], 4, 4, 64, 16, False, False),
    ([4, 2], [60, 17], 8, 2, 128, 16, True, True),         # a few rows in AIFS order
])
def test_weights(case):
    new, lens, hq, hkv, dim, page, int8, aifs = case
    pg, q, qf, perm, lse, mags, scale, group = _weights_case(*case, seed=sum(lens))
    width = max(lens) + 5
    rng = np.random.default_rng(1)
    w_in = (rng.random((len(new), hkv, width)) * 3).astype(np.float32)
    for b, n in enumerate(lens):
        w_in[b, :, max(0, n - new[b]):] = np.nan          # a new key's old entry is not read
    d_in = torch.from_numpy(w_in).to(DEV)
    w_out = torch.full((len(new), hkv, width), 9.0, device=DEV)
    dperm = None if perm is None else torch.tensor(np.concatenate(perm), dtype=torch.int32, device=DEV)
    call = lambda out, inp: B.mq_kv_weights(q.to(DEV), cu(new), pg.kv_len, pg.table, pg.cache, hq, max(new),
                                            torch.from_numpy(lse).to(DEV), out, w_in=inp, perm=dperm)
    call(w_out, d_in)
    got = w_out.cpu().numpy().astype(np.float64)
    bare = torch.zeros_like(w_out)
    call(bare, None)
    start = 0
    for b, (n, m) in enumerate(zip(new, lens)):
        assert np.all(got[b, :, m:] == 9.0)
        for g in range(hkv):
            heads = range(g * group, (g + 1) * group)
            ref = O.weights([qf[start:start + n, h] for h in heads], pg.k[b][:, g], [lse[start:start + n, h] for h in heads], scale,
                            None if perm is None else perm[b])
            ctx = max(0, m - n)
            old = np.zeros(m)
            old[:ctx] = w_in[b, g, :ctx]
            mag = max(mags[b, h] for h in heads)
            big = np.abs(lse[start:start + n][np.isfinite(lse[start:start + n])]).max(initial=0.0) + mag
            rel = (dim + 8) * 2.0 ** -23 * mag + 2.0 ** -22 * big + 2.0 ** -21 + n * group * 2.0 ** -24
            assert np.all(np.abs(got[b, g, :m] - (ref + old)) <= rel * ref + 2.0 ** -23 * (ref + old) + 1e-37)
            assert np.all(np.abs(bare[b, g, :m].cpu().numpy() - ref) <= (rel + 2.0 ** -23) * ref + 1e-37)
        start += n
    again = d_in.clone()
    call(again, again)                                     # in place: the same numbers
    for b, m in enumerate(lens):
        assert torch.equal(again[b, :, :m], w_out[b, :, :m])


def test_weights_of_many_rows_on_strided_layouts_and_graph():
    new, lens, hq, hkv, dim, page = [33, 1], [200, 90], 8, 2, 128, 16
    pg, q, qf, perm, lse, mags, scale, group = _weights_case(new, lens, hq, hkv, dim, page, False, False, 5, "token")
    pool = torch.zeros((2, 3, hkv, 256), device=DEV)
    w = pool[:, 1]                                         # sequence stride 3 * hkv * 256
    dl, qd = torch.from_numpy(lse).to(DEV), q.to(DEV)
    c = cu(new)
    run = lambda: B.mq_kv_weights(qd, c, pg.kv_len, pg.table, pg.cache, hq, 33, dl, w)
    run()
    first = w.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    w.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(w, first) and bool((pool[:, 0] == 0).all()) and bool((pool[:, 2] == 0).all())
    # a softmax row's weights sum to one
    sums = first.double().sum(-1).cpu().numpy()
    assert np.allclose(sums, np.array([[33 * group] * hkv, [group] * hkv]), rtol=1e-5)


def _evict(pg, w, budget, n_first, n_last, dst_page, dst_layout="head", same_pool=False):
    n_seq, hkv = len(pg.lens), pg.n_kv
    need = [-(-min(n, budget) // dst_page) for n in pg.lens]
    n_pages = sum(need) + 1
    rng = np.random.default_rng(2)
    order = rng.permutation(n_pages)
    dt = pg.K.dtype
    K = torch.full((n_pages, hkv, dst_page, pg.dim), 55, dtype=dt, device=DEV)
    V = torch.full((n_pages, hkv, dst_page, pg.dim), 55, dtype=dt, device=DEV)
    if dst_layout == "token":
        K, V = (x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for x in (K, V))
    table = torch.full((n_seq, max(1, -(-budget // dst_page))), -3, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = torch.from_numpy(order[at:at + n].astype(np.int32))
        at += n
    kept = torch.full((n_seq, hkv, budget), -9, dtype=torch.int32, device=DEV)
    w_out = torch.full((n_seq, hkv, budget), -9.0, device=DEV)
    new_len = torch.full((n_seq,), -9, dtype=torch.int32, device=DEV)
    dst = B.KVCache(K, V, pg.cache.k_scale, pg.cache.v_scale)
    wd = w.to(DEV)
    B.mq_kv_evict(pg.cache, pg.table, pg.kv_len, wd, budget, n_first, n_last, dst, table.to(DEV), kept, new_len, w_out=w_out)
    torch.cuda.synchronize()
    assert new_len.tolist() == [min(n, budget) for n in pg.lens]
    kept, w_out, K, V = kept.cpu().numpy(), w_out.cpu().numpy(), K.cpu(), V.cpu()
    bits = (lambda t: t.contiguous().view(torch.int16).numpy()) if dt == torch.bfloat16 else (lambda t: t.contiguous().numpy())
    used = np.zeros((n_pages, dst_page), bool)
    for b, n in enumerate(pg.lens):
        src = [pg.rows(p, b) for p in (pg.K, pg.V)]
        for g in range(hkv):
            ref = O.keep(w[b, g].numpy(), n, budget, n_first, n_last)
            assert np.array_equal(kept[b, g, :ref.size], ref)
            assert np.all(kept[b, g, ref.size:] == -9) and np.all(w_out[b, g, ref.size:] == -9.0)
            assert np.array_equal(w_out[b, g, :ref.size], w[b, g].numpy()[ref], equal_nan=True)
            i = np.arange(ref.size)
            pages = table[b].numpy()[i // dst_page]
            for pool, rows in ((K, src[0]), (V, src[1])):
                assert np.array_equal(bits(pool[pages, g, i % dst_page]), bits(rows[ref, g]))
            used[pages, i % dst_page] = True
    free = torch.from_numpy(~used)
    for pool in (K, V):
        assert bool((pool.permute(0, 2, 1, 3)[free] == 55).all())     # slots behind a sequence's new end are left alone


@pytest.mark.parametrize("lens,budget,first,last,hkv,dim,page,dst_page,int8,ties", [
    ([1], 1, 0, 0, 1, 128, 16, 16, False, False),
    ([300, 40, 41, 1], 40, 4, 10, 2, 128, 16, 64, False, False),      # one below, one at, one just above the budget
    ([5000, 700, 4096], 1024, 4, 128, 4, 128, 64, 64, False, False),
    ([5000, 4097], 129, 0, 0, 2, 64, 32, 16, True, True),
    ([900], 300, 100, 200, 2, 64, 64, 128, False, False),             # first and last fill the budget
    ([900, 10], 300, 0, 300, 2, 128, 64, 32, True, True),
    ([1500], 1499, 0, 1, 1, 128, 256, 256, False, True),
    ([100, 0, 50], 0, 0, 0, 2, 128, 16, 16, False, False),            # nothing is kept
    ([30000, 24576, 24577], 700, 4, 20, 1, 64, 128, 64, True, True),   # more keys than the selection holds in shared memory
    ([26000], 5000, 0, 0, 2, 64, 256, 32, False, False),
])
def test_evict(lens, budget, first, last, hkv, dim, page, dst_page, int8, ties):
    pg = Paged(lens, hkv, dim, page, int8, "head", 77)
    g = torch.Generator().manual_seed(3)
    w = torch.exp(2 * torch.randn((len(lens), hkv, max(lens) + 3), generator=g))
    if ties:
        w = (w * 2).round() / 2                                      # many equal weights, zeros among them
    _evict(pg, w, budget, first, last, dst_page)


def test_evict_odd_weights():
    """Zeros of both signs, infinities, NaN, denormals, negative weights, all equal."""
    lens = [400, 400, 400]
    pg = Paged(lens, 2, 128, 16, False, "token", 78)
    g = torch.Generator().manual_seed(4)
    w = torch.randn((3, 2, 400), generator=g)
    w[0, :, ::7] = float("nan")
    w[0, :, 3::7] = float("inf")
    w[0, :, 5::7] = -float("inf")
    w[1] = 0.0
    w[1, :, ::2] = -0.0
    w[2, 0] = 1e-42 * torch.arange(400)
    w[2, 1, ::3] = float("nan")
    _evict(pg, w, 333, 2, 5, 16, "token")
    _evict(pg, w, 60, 0, 0, 32)


def test_evict_within_one_pool_and_graph():
    pg = Paged([600, 350], 2, 128, 32, False, "head", 79)
    n0 = pg.K.shape[0]
    extra = 20
    K = torch.cat([pg.K, torch.zeros((extra, 2, 32, 128), dtype=torch.bfloat16, device=DEV)])
    V = torch.cat([pg.V, torch.zeros((extra, 2, 32, 128), dtype=torch.bfloat16, device=DEV)])
    cache = B.KVCache(K, V)
    table = torch.arange(n0, n0 + 14, dtype=torch.int32, device=DEV).view(2, 7)
    w = torch.rand((2, 2, 600), device=DEV)
    kept = torch.zeros((2, 2, 200), dtype=torch.int32, device=DEV)
    new_len = torch.zeros(2, dtype=torch.int32, device=DEV)
    run = lambda: B.mq_kv_evict(cache, pg.table, pg.kv_len, w, 200, 8, 32, cache, table, kept, new_len)
    run()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    w.copy_(torch.rand((2, 2, 600), device=DEV))
    g.replay()
    torch.cuda.synchronize()
    for b, n in enumerate(pg.lens):
        for h in range(2):
            ref = O.keep(w[b, h].cpu().numpy(), n, 200, 8, 32)
            assert np.array_equal(kept[b, h].cpu().numpy(), ref)
            i = torch.arange(200)
            got = K[table[b, (i // 32).to(DEV)].long(), h, (i % 32).to(DEV)].cpu()
            assert torch.equal(got, pg.rows(pg.K, b)[torch.from_numpy(ref), h])


def test_evict_bad_pages():
    """A source page outside the cache reads as zeros, a destination page outside it is not written."""
    pg = Paged([100], 1, 128, 16, False, "head", 80)
    pg.table[0, 1] = 1000
    K, V = (torch.full((2, 1, 16, 128), 55.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    table = torch.tensor([[1, 4, 0]], dtype=torch.int32, device=DEV)
    kept = torch.zeros((1, 1, 48), dtype=torch.int32, device=DEV)
    new_len = torch.zeros(1, dtype=torch.int32, device=DEV)
    w = torch.zeros((1, 1, 100), device=DEV)               # all equal: the first 48 stay
    B.mq_kv_evict(pg.cache, pg.table, pg.kv_len, w, 48, 0, 0, B.KVCache(K, V), table, kept, new_len)
    torch.cuda.synchronize()
    assert kept.flatten().tolist() == list(range(48))
    rows = torch.from_numpy(pg.k[0]).to(torch.bfloat16)
    assert torch.equal(K[1, 0].cpu(), rows[:16, 0]) and torch.equal(K[0, 0].cpu(), rows[32:48, 0])


def test_odd_weight_pitch():
    """Weights whose rows start on any 4-byte boundary."""
    pg = Paged([77, 130], 3, 64, 16, False, "head", 81)
    w = torch.rand((2, 3, 131), generator=torch.Generator().manual_seed(1))
    _evict(pg, w, 50, 1, 3, 16)


@pytest.mark.parametrize("new,lens,hq", [([1, 1], [90, 30], 4), ([40, 3], [300, 30], 8)])
def test_weight_rows_shorter_than_a_sequence(new, lens, hq):
    """Keys behind the row of the weights are neither read nor written, and reported; the others keep their values."""
    pg, q, qf, perm, lse, mags, scale, group = _weights_case(new, lens, hq, 2, 128, 16, False, False, 90)
    full = torch.zeros((2, 2, max(lens)), device=DEV)
    args = (q.to(DEV), cu(new), pg.kv_len, pg.table, pg.cache, hq, max(new), torch.from_numpy(lse).to(DEV))
    B.mq_kv_weights(*args, full)
    keys = 37
    for w_in in (False, True):
        pool = torch.full((2, 2, 64), 7.0, device=DEV)
        w = pool[:, :, 10:10 + keys]
        status = torch.zeros(2, dtype=torch.int32, device=DEV)
        B.mq_kv_weights(*args, w, w_in=w if w_in else None, status=status)
        assert status[0].item() == B.MQ_ERR_INVALID_ARG
        assert bool((pool[:, :, :10] == 7).all()) and bool((pool[:, :, 10 + keys:] == 7).all())
        for b, n in enumerate(lens):
            m, ctx = min(n, keys), min(n - new[b], keys)
            want = full[b, :, :m].clone()
            if w_in:
                want[:, :ctx] += 7.0
            assert torch.equal(w[b, :, :m], want) and bool((w[b, :, m:] == 7).all())
    status = torch.zeros(2, dtype=torch.int32, device=DEV)
    B.mq_kv_weights(*args, full, status=status)            # rows of just the longest length are long enough
    assert status.tolist() == [0, 0]


def test_weights_without_rows_copies():
    pg = Paged([20, 70], 2, 128, 16)
    w_in = torch.rand((2, 2, 70), device=DEV)
    none = torch.zeros(3, dtype=torch.int32, device=DEV)
    q, lse = torch.empty((0, 512), dtype=torch.bfloat16, device=DEV), torch.empty((0, 4), device=DEV)
    for inp in (w_in, None):
        w = torch.full((2, 2, 70), 9.0, device=DEV)
        B.mq_kv_weights(q, none, pg.kv_len, pg.table, pg.cache, 4, 0, lse, w, w_in=inp)
        for b, n in enumerate(pg.lens):
            assert torch.equal(w[b, :, :n], w_in[b, :, :n] if inp is not None else torch.zeros((2, n), device=DEV))
            assert bool((w[b, :, n:] == 9).all())


@pytest.mark.parametrize("lens,budget", [([100], 60), ([30000], 500), ([50], 60)])
def test_evict_with_weight_rows_shorter_than_a_sequence(lens, budget):
    """Keys behind the row of the weights count as NaN: they stay only where no others are left, or as the last ones."""
    pg = Paged(lens, 1, 64, 64, False, "head", 91)
    n, keys = lens[0], 45
    w = torch.rand((1, 1, 64), generator=torch.Generator().manual_seed(2)).to(DEV)[:, :, :keys]
    K, V = (torch.zeros((8, 1, 64, 64), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    table = torch.arange(8, dtype=torch.int32, device=DEV)[None]
    kept = torch.zeros((1, 1, budget), dtype=torch.int32, device=DEV)
    new_len = torch.zeros(1, dtype=torch.int32, device=DEV)
    w_out = torch.full((1, 1, budget), 3.0, device=DEV)
    B.mq_kv_evict(pg.cache, pg.table, pg.kv_len, w, budget, 0, 2, B.KVCache(K, V), table, kept, new_len, w_out=w_out)
    m = min(n, budget)
    want = list(range(n)) if n <= budget else list(range(budget - 2)) + [n - 2, n - 1]
    assert new_len.item() == m and kept[0, 0, :m].tolist() == want
    assert torch.equal(w_out[0, 0, :keys], w[0, 0]) and bool(torch.isnan(w_out[0, 0, keys:m]).all())


@pytest.mark.parametrize("int8", [False, True])
def test_far_pages_give_the_same_as_near_ones(int8):
    """Pages behind 2^32 bytes: every call gives the bits that it gives on a packed pool."""
    hq, hkv, dim, page, lens = 8, 2, 128, 16, [70, 33]
    pg = Paged(lens, hkv, dim, page, int8, "head", 95)
    n = pg.K.shape[0]
    stride = (1 << 32) // pg.K.element_size() // (n - 2)      # the last pages start behind 2^32 bytes
    stride -= stride % 16
    far = []
    for pool in (pg.K, pg.V):
        big = torch.empty((n - 1) * stride + hkv * page * dim, dtype=pool.dtype, device=DEV)
        view = big.as_strided((n, hkv, page, dim), (stride, page * dim, dim, 1))
        view.copy_(pool)
        far.append(view)
    assert (n - 1) * stride * pg.K.element_size() > 1 << 32
    caches = [pg.cache, B.KVCache(*far, pg.cache.k_scale, pg.cache.v_scale)]
    g = torch.Generator().manual_seed(3)
    for new in ([1, 1], [30, 7]):
        q = torch.randn((sum(new), hq * dim), generator=g).to(torch.bfloat16).to(DEV)
        got = []
        for cache in caches:
            ws = B.new_kv_attention_workspace(2, sum(new), max(new), pg.table.shape[1], hq, cache)
            o, lse, w = torch.empty_like(q), torch.empty((sum(new), hq), device=DEV), torch.zeros((2, hkv, max(lens)), device=DEV)
            B.mq_kv_attention(q, cu(new), pg.kv_len, pg.table, cache, hq, max(new), o, ws, lse=lse)
            B.mq_kv_weights(q, cu(new), pg.kv_len, pg.table, cache, hq, max(new), lse, w)
            K, V = (torch.zeros((4, hkv, page, dim), dtype=pg.K.dtype, device=DEV) for _ in range(2))
            table = torch.tensor([[2, 0], [1, 3]], dtype=torch.int32, device=DEV)
            kept, length = torch.zeros((2, hkv, 32), dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
            B.mq_kv_evict(cache, pg.table, pg.kv_len, w, 32, 2, 3, B.KVCache(K, V, cache.k_scale, cache.v_scale), table, kept, length)
            torch.cuda.synchronize()
            assert B.mq_last_device_status(ws) == (B.MQ_OK, 0)
            got.append((o, lse, w, kept, K, V))
        assert all(torch.equal(a, b) for a, b in zip(*got)) and bool(torch.isfinite(got[0][0]).all())


@pytest.mark.parametrize("new,lens,hq,int8", [([1, 1], [90, 30], 4, False), ([10, 9], [300, 130], 8, False), ([10, 9], [300, 130], 8, True), ([40, 3], [200, 60], 14, False)])
def test_rows_that_are_nan_stay_with_their_sequence(new, lens, hq, int8):
    """The rows of the sequence behind lie in the same tile of queries."""
    pg, q, qf, perm, lse, mags, scale, group = _weights_case(new, lens, hq, 2, 128, 16, int8, False, 96)
    got = []
    for bad in (False, True):
        rows, l = q.clone(), torch.from_numpy(lse.copy())
        if bad:
            rows[new[0]:] = float("nan")
            l[new[0]:] = float("nan")
        w = torch.zeros((2, 2, max(lens)), device=DEV)
        B.mq_kv_weights(rows.to(DEV), cu(new), pg.kv_len, pg.table, pg.cache, hq, max(new), l.to(DEV), w)
        got.append(w)
    assert torch.equal(got[0][0], got[1][0]) and bool(torch.isnan(got[1][1, :, 0]).all())


@pytest.mark.parametrize("budget", [700, 64, 0])
def test_evict_with_lengths_in_place(budget):
    """new_len may be kv_len: no head may see the new length instead of the old one."""
    rng = np.random.default_rng(8)
    hkv, dim, page = 8, 64, 16
    lens = [int(x) for x in rng.integers(1, 1500, 24)] + [0, budget, budget + 1]
    pg = Paged(lens, hkv, dim, page, True, "head", 97)
    w = torch.rand((len(lens), hkv, max(lens)), generator=torch.Generator().manual_seed(6)).to(DEV)
    width = max(1, -(-budget // page))
    table = torch.arange(len(lens) * width, dtype=torch.int32, device=DEV).view(len(lens), width)
    K, V = (torch.zeros((len(lens) * width, hkv, page, dim), dtype=torch.int8, device=DEV) for _ in range(2))
    dst = B.KVCache(K, V, pg.cache.k_scale, pg.cache.v_scale)
    kept = torch.full((len(lens), hkv, budget), -9, dtype=torch.int32, device=DEV)
    for _ in range(3):
        kept.fill_(-9)
        length = pg.kv_len.clone()
        B.mq_kv_evict(pg.cache, pg.table, length, w, budget, 2, 3, dst, table, kept, length) if budget else \
            B.mq_kv_evict(pg.cache, pg.table, length, w, budget, 0, 0, dst, table, kept, length)
        assert length.tolist() == [min(n, budget) for n in lens]
        for b, n in enumerate(lens if budget else []):
            for g in range(hkv):
                ref = O.keep(w[b, g].cpu().numpy(), n, budget, 2, 3)
                assert np.array_equal(kept[b, g, :ref.size].cpu().numpy(), ref) and bool((kept[b, g, ref.size:] == -9).all())
