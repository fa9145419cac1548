"""mq_kv_attention against the float64 definition.

Tolerances (derived, per element): the bf16 output is off by half a step, 2^-8 |o|; a probability enters the second
product off by half a step of its type (2^-8 bf16, 2^-11 fp16) and by its own error, which is that of its score -- a
float32 sum of D exact products, at most (D + 8) 2^-23 of the sum of their magnitudes -- plus a few float32 roundings
of the exponent's argument and of exp2 (2^-19 together); all of them are relative to sum_j p |v|.  An fp16 probability
below fp16's normal range is off by half its smallest step, 2^-25, whatever its size; as the largest of a row is at least
2^6 there (2^14 in the kernel for few rows), that is at most 2^-31 (2^-39) of the softmax's denominator per key, times |v|.
"""
import numpy as np
import pytest
import torch

from oracle import kv_oracle as O
from paper_2502_00425_b200 import binding as B

from kv_util import DEV, Paged, aifs_perm, cu

pytestmark = pytest.mark.gpu


def _inputs(new, lens, hq, hkv, dim, page, int8, layout, seed, q_scale=1.2, extra_pages=2):
    pg = Paged(lens, hkv, dim, page, int8, layout, seed, extra_pages)
    g = torch.Generator().manual_seed(seed + 1)
    q = (torch.randn((sum(new), hq * dim), generator=g) * q_scale).to(torch.bfloat16)
    return pg, q


def _run(pg, q, new, hq, perm=None, max_q=None, lse=True, scale=None, pad_cols=0, ws=None):
    total = sum(new)
    dim = pg.dim
    wide = torch.zeros((total + 3, hq * dim + pad_cols), dtype=torch.bfloat16, device=DEV)
    wide[:total, :hq * dim] = q.to(DEV)
    o_full = torch.full((total + 3, hq * dim + pad_cols), 7.0, dtype=torch.bfloat16, device=DEV)
    lse_full = torch.full((total + 3, hq), 7.0, device=DEV)
    qd, od = wide[:total, :hq * dim], o_full[:total, :hq * dim]
    max_q = max(new + [0]) if max_q is None else max_q
    if ws is None:
        ws = B.new_kv_attention_workspace(len(new), total, max_q, pg.table.shape[1], hq, pg.cache)
    dperm = None if perm is None else torch.tensor(np.concatenate(perm), dtype=torch.int32, device=DEV)
    B.mq_kv_attention(qd, cu(new), pg.kv_len, pg.table, pg.cache, hq, max_q, od, ws, lse=lse_full[:total] if lse else None,
                      perm=dperm, scale=scale)
    torch.cuda.synchronize()
    assert B.mq_last_device_status(ws) == (B.MQ_OK, 0)
    assert bool((o_full[total:] == 7.0).all()) and bool((lse_full[total:] == 7.0).all())   # rows behind the last sequence
    if pad_cols:
        assert bool((o_full[:, hq * dim:] == 7.0).all())
    return od.float().cpu().numpy().astype(np.float64), lse_full[:total].cpu().numpy().astype(np.float64)


def _check(pg, q, new, hq, o, lse, perm=None, scale=None, seqs=None, heads=None):
    hkv, dim = pg.n_kv, pg.dim
    group = hq // hkv
    scale = dim ** -0.5 if scale is None else scale
    qf = q.double().numpy().reshape(-1, hq, dim)
    p_step = 2.0 ** -11 if pg.int8 else 2.0 ** -8
    start = 0
    worst = 0.0
    for b, n in enumerate(new):
        if seqs is None or b in seqs:
            for h in (range(hq) if heads is None else heads):
                g = h // group
                ref, ref_lse, _, abs_pv, mag = O.attention(qf[start:start + n, h], pg.k[b][:, g], pg.v[b][:, g], scale,
                                                           None if perm is None else perm[b])
                got = o[start:start + n, h * dim:(h + 1) * dim]
                ds = (dim + 8) * 2.0 ** -23 * mag[:, None]
                tol = 2.0 ** -8 * np.abs(ref) + (p_step + 2 * ds + 2.0 ** -19) * abs_pv + 1e-30
                if pg.int8:
                    few = max(new) * group <= 32
                    tol = tol + 2.0 ** (-39 if few else -31) * np.abs(pg.v[b][:, g]).sum(0)
                assert np.isfinite(got).all()
                worst = max(worst, float((np.abs(got - ref) / tol).max(initial=0.0)))
                got_l = lse[start:start + n, h]
                dead = np.isneginf(ref_lse)
                assert np.array_equal(dead, np.isneginf(got_l))
                tol_l = ds[:, 0] + 2.0 ** -20 * (1 + np.abs(ref_lse))
                assert np.all(np.abs(got_l[~dead] - ref_lse[~dead]) <= tol_l[~dead])
        start += n
    assert worst <= 1.0, worst


CASES = [
    # new tokens per sequence, total keys per sequence, hq, hkv, dim, page, int8, aifs
    ([1], [1], 2, 2, 128, 16, False, False),                                   # the first token of a sequence
    ([1], [3361], 28, 4, 128, 64, False, False),                               # one sequence split over many CTAs
    ([1, 1, 1, 1, 1], [1, 16, 17, 700, 64], 32, 8, 128, 16, False, False),     # ragged, tiles and pages that end exactly
    ([1] * 9, [5, 300, 40, 129, 65, 1, 2, 513, 1200], 8, 1, 64, 32, False, False),
    ([1, 1, 1], [33, 1025, 450], 14, 2, 128, 64, True, False),
    ([1, 1, 1], [33, 1025, 450], 16, 2, 64, 16, True, False),
    ([3, 1, 0, 2], [100, 1, 50, 777], 28, 4, 128, 64, False, False),           # a sequence without new tokens
    ([5, 33], [5, 160], 4, 2, 128, 16, False, False),                          # a whole prompt; a chunk behind a context
    ([70, 1, 129], [70, 900, 400], 28, 4, 128, 128, False, False),
    ([129, 40], [300, 40], 8, 4, 64, 64, False, False),
    ([65, 200], [330, 200], 14, 2, 128, 32, True, False),
    ([65, 31], [130, 95], 6, 2, 64, 256, True, False),
    ([40, 150], [240, 150], 8, 2, 128, 64, False, True),                       # AIFS order, behind a context and without one
    ([50, 3, 1], [250, 3, 90], 12, 4, 64, 16, False, True),
    ([77], [500], 28, 4, 128, 64, True, True),
    ([10, 4], [6, 0], 4, 2, 128, 16, False, False),                            # fewer keys than rows: some rows see nothing
    ([130], [100], 4, 2, 128, 16, False, False),
    ([10], [6], 4, 1, 64, 16, True, False),
    ([2], [19], 130, 1, 128, 16, False, False),                                # more query heads per key/value head than a block has rows
    ([300], [1300], 7, 1, 128, 64, False, False),                              # several row blocks, uneven group
    ([257, 128, 1, 64], [257, 1000, 2000, 64], 32, 8, 128, 64, False, False),  # a mixed batch
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention(case):
    new, lens, hq, hkv, dim, page, int8, aifs = CASES[case]
    rng = np.random.default_rng(case)
    pg, q = _inputs(new, lens, hq, hkv, dim, page, int8, "head", 100 + case)
    perm = aifs_perm(rng, new) if aifs else None
    o, lse = _run(pg, q, new, hq, perm)
    heads = None if hq <= 8 else sorted({0, hq // hkv - 1, hq - 1, hq // 2})
    _check(pg, q, new, hq, o, lse, perm, heads=heads)


@pytest.mark.parametrize("layout", ["token", "padded"])
@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("new,lens", [([1, 1], [90, 1111]), ([100, 7], [180, 300])])
def test_layouts_and_row_pitches(layout, int8, new, lens):
    pg, q = _inputs(new, lens, 12, 4, 128, 32, int8, layout, 7)
    o, lse = _run(pg, q, new, 12, pad_cols=24)
    _check(pg, q, new, 12, o, lse, heads=[0, 5, 11])


def test_scale_and_no_lse_and_loose_bounds():
    new, lens = [1, 2, 30], [40, 300, 77]
    pg, q = _inputs(new, lens, 8, 2, 128, 16, False, "head", 11, extra_pages=9)
    o, lse = _run(pg, q, new, 8, scale=0.31)
    _check(pg, q, new, 8, o, lse, scale=0.31)
    o2, _ = _run(pg, q, new, 8, scale=0.31, lse=False)
    assert np.array_equal(o, o2)
    o3, lse3 = _run(pg, q, new, 8, scale=0.31, max_q=33)   # bounds above the lengths: allowed; the split may differ
    _check(pg, q, new, 8, o3, lse3, scale=0.31)


@pytest.mark.parametrize("int8", [False, True])
def test_large_scores_and_one_hot_rows(int8):
    """Scores of a few hundred: the softmax is one-hot and the maximum moves over the whole range."""
    new, lens = [2, 40], [500, 700]
    pg, q = _inputs(new, lens, 8, 2, 128, 64, int8, "head", 12, q_scale=40.0)
    o, lse = _run(pg, q, new, 8)
    _check(pg, q, new, 8, o, lse)


def test_query_magnitudes_over_the_whole_range_on_an_int8_cache():
    """Rows of very large and very small magnitude keep their bits in the fp16 product."""
    new, lens = [4], [200]
    pg, q = _inputs(new, lens, 4, 2, 128, 16, True, "head", 13)
    mult = torch.tensor([1e-6, 1.0, 3e4, 0.0])
    q = (q.float() * mult[:, None]).to(torch.bfloat16)
    o, lse = _run(pg, q, new, 4, scale=1e-4)
    _check(pg, q, new, 4, o, lse, scale=1e-4)


@pytest.mark.parametrize("aifs", [False, True])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
@pytest.mark.parametrize("n_new,n_all,hq,hkv", [(20, 60, 4, 2), (150, 400, 8, 2)])
def test_values_a_row_does_not_see_do_not_reach_it(value, aifs, n_new, n_all, hq, hkv):
    """An infinite (or NaN) key and value in the chunk: rows that see it are not finite, all others are exact."""
    new, lens = [n_new], [n_all]
    pg, q = _inputs(new, lens, hq, hkv, 128, 16, False, "head", 14)
    perm = aifs_perm(np.random.default_rng(3), new) if aifs else None
    bad = n_all - n_new // 3
    page, slot = int(pg.table[0, bad // 16]), bad % 16
    pg.V[page, :, slot] = value
    pg.v[0][bad] = value
    if np.isnan(value):
        pg.K[page, :, slot] = value
        pg.k[0][bad] = 0.0
    o, lse = _run(pg, q, new, hq, perm)
    see = O.visible(n_new, n_all, None if perm is None else perm[0])[:, bad]
    assert see.any() and not see.all()
    assert not np.isfinite(o[see]).any()
    rows = np.flatnonzero(~see)
    clean = Paged(lens, hkv, 128, 16, False, "head", 14)
    dim, group = 128, hq // hkv
    qf = q.double().numpy().reshape(-1, hq, dim)
    for h in range(hq):
        ref, _, _, abs_pv, mag = O.attention(qf[:, h], clean.k[0][:, h // group], clean.v[0][:, h // group], dim ** -0.5,
                                             None if perm is None else perm[0])
        tol = 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2 * (dim + 8) * 2.0 ** -23 * mag[:, None] + 2.0 ** -19) * abs_pv
        assert np.all(np.abs(o[:, h * dim:(h + 1) * dim] - ref)[rows] <= tol[rows])


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("new,lens", [([1, 1], [100, 50]), ([40, 1], [100, 50])])
def test_bad_page_numbers_read_as_zeros_and_are_reported(int8, new, lens):
    pg, q = _inputs(new, lens, 4, 2, 128, 16, int8, "head", 15)
    pg.table[0, 2] = pg.K.shape[0] + 3
    pg.table[0, 4] = -2
    for x in (pg.k[0], pg.v[0]):
        x[32:48] = 0.0
        x[64:80] = 0.0
    ws = B.new_kv_attention_workspace(2, sum(new), max(new), pg.table.shape[1], 4, pg.cache)
    o = torch.empty((sum(new), 512), dtype=torch.bfloat16, device=DEV)
    lse = torch.empty((sum(new), 4), device=DEV)
    B.mq_kv_attention(q.to(DEV), cu(new), pg.kv_len, pg.table, pg.cache, 4, max(new), o, ws, lse=lse)
    torch.cuda.synchronize()
    assert B.mq_last_device_status(ws)[0] == B.MQ_ERR_INVALID_ARG
    _check(pg, q, new, 4, o.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64))


@pytest.mark.parametrize("new_a,lens_a,new_b,lens_b", [([1, 1, 1], [700, 90, 16], [1, 1, 1], [20, 1100, 333]),
                                                       ([50, 60, 1], [300, 60, 80], [64, 1, 46], [64, 1024, 46])])
def test_captured_graph_follows_new_lengths(new_a, lens_a, new_b, lens_b):
    """A captured call replayed after the lengths, the table and the queries changed on the device; two graphs share a workspace."""
    hq, hkv, dim, page = 8, 2, 128, 16
    width = 80
    total = sum(new_a)
    assert total == sum(new_b)
    pa, qa = _inputs(new_a, lens_a, hq, hkv, dim, page, False, "head", 21)
    pb, qb = _inputs(new_b, lens_b, hq, hkv, dim, page, False, "head", 22)
    n_pages = max(pa.K.shape[0], pb.K.shape[0])
    K = torch.zeros((n_pages, hkv, page, dim), dtype=torch.bfloat16, device=DEV)
    V = torch.zeros_like(K)
    cache = B.KVCache(K, V)
    table = torch.zeros((3, width), dtype=torch.int32, device=DEV)
    kv_len, cu_q = torch.zeros(3, dtype=torch.int32, device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV)
    q = torch.zeros((total, hq * dim), dtype=torch.bfloat16, device=DEV)
    outs = [(torch.zeros_like(q), torch.zeros((total, hq), device=DEV)) for _ in range(2)]
    max_q = max(new_a + new_b)
    ws = B.new_kv_attention_workspace(3, total, max_q, width, hq, cache)

    def load(pg, qq, new):
        K[:pg.K.shape[0]], V[:pg.V.shape[0]] = pg.K, pg.V
        table.fill_(-1)
        table[:, :pg.table.shape[1]] = pg.table
        kv_len.copy_(pg.kv_len)
        cu_q.copy_(cu(new))
        q.copy_(qq.to(DEV))

    load(pa, qa, new_a)
    call = lambda o, lse: B.mq_kv_attention(q, cu_q, kv_len, table, cache, hq, max_q, o, ws, lse=lse)
    call(*outs[0])
    torch.cuda.synchronize()
    graphs = []
    for o, lse in outs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(o, lse)
        graphs.append(g)
    for pg, qq, new in ((pa, qa, new_a), (pb, qb, new_b), (pa, qa, new_a)):
        load(pg, qq, new)
        for o, lse in outs:
            o.fill_(0.0)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert B.mq_last_device_status(ws)[0] == B.MQ_OK
        for o, lse in outs:
            _check(pg, qq, new, hq, o.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64), heads=[0, 7])


def test_results_do_not_depend_on_timing():
    new, lens = [1, 1, 30], [2500, 90, 700]
    pg, q = _inputs(new, lens, 28, 4, 128, 64, False, "head", 30)
    first = _run(pg, q, new, 28)
    for _ in range(4):
        again = _run(pg, q, new, 28)
        assert np.array_equal(first[0], again[0]) and np.array_equal(first[1], again[1])


def test_two_streams_with_their_own_workspaces():
    cases = [([1, 1], [1500, 300], 40), ([80], [500], 41)]
    made = []
    for new, lens, seed in cases:
        pg, q = _inputs(new, lens, 8, 2, 128, 64, False, "head", seed)
        ws = B.new_kv_attention_workspace(len(new), sum(new), max(new), pg.table.shape[1], 8, pg.cache)
        made.append((pg, q, new, ws, cu(new), q.to(DEV), torch.empty_like(q, device=DEV), torch.empty((sum(new), 8), device=DEV)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in made]
    for _ in range(5):
        for st, (pg, q, new, ws, c, qd, o, lse) in zip(streams, made):
            with torch.cuda.stream(st):
                B.mq_kv_attention(qd, c, pg.kv_len, pg.table, pg.cache, 8, max(new), o, ws, lse=lse)
    torch.cuda.synchronize()
    for pg, q, new, ws, c, qd, o, lse in made:
        _check(pg, q, new, 8, o.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64), heads=[0, 7])


@pytest.mark.parametrize("new", [[1, 1], [40, 3]])
def test_a_cache_without_pages_reads_as_zeros(new):
    """No page exists: every page number is outside the cache (and reported), keys and values are zeros."""
    K = torch.empty((0, 2, 16, 128), dtype=torch.bfloat16, device=DEV)
    cache = B.KVCache(K, K.clone())
    table = torch.zeros((2, 4), dtype=torch.int32, device=DEV)
    lens = torch.tensor([50, 40], dtype=torch.int32, device=DEV)
    q = torch.randn((sum(new), 512), device=DEV).to(torch.bfloat16)
    o, lse = torch.full_like(q, 7.0), torch.zeros((sum(new), 4), device=DEV)
    ws = B.new_kv_attention_workspace(2, sum(new), max(new), 4, 4, cache)
    B.mq_kv_attention(q, cu(new), lens, table, cache, 4, max(new), o, ws, lse=lse)
    w = torch.full((2, 2, 64), 9.0, device=DEV)
    B.mq_kv_weights(q, cu(new), lens, table, cache, 4, max(new), lse, w)
    torch.cuda.synchronize()
    assert B.mq_last_device_status(ws)[0] == B.MQ_ERR_INVALID_ARG
    assert bool((o == 0).all())
    counts = torch.cat([torch.arange(n - k + 1, n + 1) for k, n in zip(new, (50, 40))]).double()   # keys that a row sees
    assert torch.allclose(lse.double().cpu(), counts.log()[:, None].expand(-1, 4), atol=1e-5)
    assert torch.allclose(w.double().sum(-1).cpu(), torch.tensor([[2.0 * new[0]] * 2, [2.0 * new[1]] * 2]).double() + torch.tensor([[9.0 * 14], [9.0 * 24]]), atol=1e-4)


@pytest.mark.parametrize("new_most", [1, 20])
def test_the_most_sequences_of_a_call(new_most):
    """2048 sequences, some without keys or without new tokens, lengths below and above one tile."""
    rng = np.random.default_rng(5)
    new = [int(x) for x in rng.integers(0, new_most + 1, 2048)]
    lens = [int(x) + n for x, n in zip(rng.integers(0, 70, 2048), new)]
    pg, q = _inputs(new, lens, 4, 2, 64, 16, False, "head", 50)
    o, lse = _run(pg, q, new, 4)
    _check(pg, q, new, 4, o, lse, seqs=set(range(0, 2048, 17)) | {2047}, heads=[0, 3])
    w = torch.zeros((2048, 2, max(lens)), device=DEV)
    B.mq_kv_weights(q.to(DEV), cu(new), pg.kv_len, pg.table, pg.cache, 4, max(new), torch.from_numpy(lse.astype(np.float32)).to(DEV), w)
    sums = w.double().sum(-1).cpu().numpy()
    assert np.allclose(sums, np.array(new)[:, None] * 2.0 * np.ones((1, 2)), rtol=2e-5, atol=1e-6)   # every row hands out weight 1


def test_empty_calls_are_no_ops():
    pg = Paged([20], 2, 128, 16)
    ws = B.new_kv_attention_workspace(1, 1, 1, pg.table.shape[1], 4, pg.cache)
    q = torch.empty((0, 512), dtype=torch.bfloat16, device=DEV)
    B.mq_kv_attention(q, cu([0]), pg.kv_len, pg.table, pg.cache, 4, 0, q, ws)
    empty = torch.empty(0, dtype=torch.int32, device=DEV)
    B.mq_kv_attention(q, torch.zeros(1, dtype=torch.int32, device=DEV), empty, empty.view(0, 1), pg.cache, 4, 0, q, ws)
    torch.cuda.synchronize()


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("new,lens,hq,hkv", [([1, 1], [40, 3361], 8, 2), ([3], [900], 8, 2), ([40, 300], [300, 5000], 8, 2), ([9], [12000], 28, 4)])
def test_a_query_that_is_nan_gives_nan_and_reaches_no_other(int8, new, lens, hq, hkv):
    """Also where its keys are spread over several workers."""
    pg, q = _inputs(new, lens, hq, hkv, 128, 64, int8, "head", 61)
    clean, clean_lse = _run(pg, q, new, hq)
    bad = [(0, 1), (sum(new) - 1, hq - 1), (sum(new) // 2, 0)]
    for i, h in bad:
        q[i, h * 128:(h + 1) * 128] = float("nan")
    q[0, 0] = float("nan")                                  # a single channel is enough
    o, lse = _run(pg, q, new, hq)
    hit = np.zeros((sum(new), hq), bool)
    for i, h in bad + [(0, 0)]:
        hit[i, h] = True
    o, clean = o.reshape(-1, hq, 128), clean.reshape(-1, hq, 128)
    assert np.isnan(o[hit]).all() and np.isnan(lse[hit]).all()
    assert np.array_equal(o[~hit], clean[~hit]) and np.array_equal(lse[~hit], clean_lse[~hit])


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("new,lens,hq,hkv", [([13, 30], [3000, 900], 28, 4), ([36, 20], [2600, 2500], 14, 2), ([50, 17], [3500, 64], 4, 4)])
def test_results_do_not_depend_on_the_sequence_behind(int8, new, lens, hq, hkv):
    """The last block of a sequence's rows is filled up with the next sequence's tokens: however large those are, the first
    sequence keeps its bits."""
    pg, q = _inputs(new, lens, hq, hkv, 128, 64, int8, "head", 71)
    first = []
    for factor in (1.0, 0.0, 3.0, 100.0):
        rows = q.clone()
        rows[new[0]:] = (rows[new[0]:].float() * factor).to(torch.bfloat16)
        o, lse = _run(pg, rows, new, hq)
        _check(pg, rows, new, hq, o, lse, seqs={0}, heads=[0, hq - 1])
        first.append((o[:new[0]], lse[:new[0]]))
    for o, lse in first[1:]:
        assert np.array_equal(o, first[0][0]) and np.array_equal(lse, first[0][1])


def test_results_do_not_depend_on_the_calls_before():
    """A group of 7 fills 126 of a block's 128 query rows; what other kernels leave in shared memory must not matter."""
    new, lens, hq = [200, 40], [3000, 1500], 28
    pg, q = _inputs(new, lens, hq, 4, 128, 64, False, "head", 72)
    big, qb = _inputs([300], [2000], 8, 2, 128, 64, False, "head", 73, q_scale=200.0)
    first = _run(pg, q, new, hq)
    _check(pg, q, new, hq, *first, heads=[0, 27])
    for scale in (1.0, 50.0, float("nan")):
        o, lse = _run(big, (qb.float() * scale).to(torch.bfloat16), [300], 8)
        w = torch.zeros((1, 2, 2000), device=DEV)
        B.mq_kv_weights((qb.float() * scale).to(torch.bfloat16).to(DEV), cu([300]), big.kv_len, big.table, big.cache, 8, 300,
                        torch.from_numpy(lse.astype(np.float32)).to(DEV), w)
        again = _run(pg, q, new, hq)
        assert np.array_equal(first[0], again[0]) and np.array_equal(first[1], again[1])


@pytest.mark.parametrize("new,lens", [([1, 2], [40, 300]), ([40, 200], [200, 900]), ([90], [60])])
@pytest.mark.parametrize("aifs", [False, True])
@pytest.mark.parametrize("value", [0.0, -0.0125, 1e-42])
def test_static_scales_that_are_not_positive(value, new, lens, aifs):
    """Zero (a head whose keys were all zero when its scale was taken: its softmax is uniform over what a row sees), a
    negative number, and one below the normal range."""
    pg, q = _inputs(new, lens, 6, 3, 128, 16, True, "head", 74)
    old = float(pg.k_scale[1])
    pg.cache.k_scale[1] = value
    for k in pg.k:
        k[:, 1] = np.round(k[:, 1] / old) * float(np.float32(value))
    perm = aifs_perm(np.random.default_rng(4), new) if aifs else None
    o, lse = _run(pg, q, new, 6, perm)
    _check(pg, q, new, 6, o, lse, perm)


@pytest.mark.parametrize("new,lens,hq,hkv,dim", [([1, 2], [70, 500], 4, 2, 128), ([1], [2100], 12, 1, 64), ([16], [64], 1, 1, 128)])
def test_a_query_channel_that_dwarfs_the_others_on_an_int8_cache(new, lens, hq, hkv, dim):
    """One channel 2^20 times the others, and the keys have nothing there: the small channels alone decide, so they need their
    bits.  (What fp16 loses of them, 2^-39 of the largest = 2^-19 per channel, is within the tolerance for the sum's own
    roundings: (D + 8) 2^-23 of sum |q| |k|, with |q| about 1.)  The weights take the same queries."""
    pg, q = _inputs(new, lens, hq, hkv, dim, 16, True, "head", 75)
    q[:, ::dim] = 2.0 ** 20
    pg.K[:, :, :, 0] = 0
    for k in pg.k:
        k[:, :, 0] = 0.0
    o, lse = _run(pg, q, new, hq)
    _check(pg, q, new, hq, o, lse)
    w = torch.zeros((len(new), hkv, max(lens)), device=DEV)
    B.mq_kv_weights(q.to(DEV), cu(new), pg.kv_len, pg.table, pg.cache, hq, max(new), torch.from_numpy(lse.astype(np.float32)).to(DEV), w)
    qf, group, start = q.double().numpy().reshape(-1, hq, dim), hq // hkv, 0
    for b, n in enumerate(new):
        for g in range(hkv):
            heads = range(g * group, (g + 1) * group)
            rows = [qf[start:start + n, h] for h in heads]
            ref = O.weights(rows, pg.k[b][:, g], [lse[start:start + n, h] for h in heads], dim ** -0.5)
            mag = max(O.attention(r, pg.k[b][:, g], pg.v[b][:, g], dim ** -0.5)[4].max() for r in rows)
            rel = (dim + 8) * 2.0 ** -23 * mag + 2.0 ** -22 * (mag + np.abs(lse).max()) + 2.0 ** -21 + n * group * 2.0 ** -24
            assert np.all(np.abs(w[b, g, :lens[b]].double().cpu().numpy() - ref) <= (rel + 2.0 ** -23) * ref + 1e-37)
        start += n
