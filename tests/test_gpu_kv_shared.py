"""mq_kv_attention_shared against the float64 definition, every sequence by its own list of keys.

Tolerances: those of mq_kv_attention's tests (derived there), with the fp16 floor of the chunk kernel for any int8 cache, as the shared keys may go
through it, and 2^-20 more for the join of the two lists (its factors are exponentials of float32 differences).
"""
import numpy as np
import pytest
import torch

from oracle import kv_oracle as O
from paper_2502_00425_b200 import binding as B

from kv_util import DEV, aifs_perm, cu

pytestmark = pytest.mark.gpu


class Groups:
    """Sequences in groups: groups[i] = (keys in common, [keys of its own of every sequence]).  Slots behind a sequence's end hold NaN (bf16) or
    extreme codes, table entries behind its last page numbers outside the cache.  Only whole pages are the same in memory."""

    def __init__(self, groups, n_kv, dim, page, int8=False, token_layout=False, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.page, self.int8, self.n_kv, self.dim = page, int8, n_kv, dim
        self.lens, self.leader, self.shared = [], [], []
        plan = []                                    # per sequence: (rows in common, rows of its own)
        rand = lambda n: torch.randn((n, n_kv, dim), generator=g)
        for common, own in groups:
            first, k0, v0 = len(self.lens), rand(common), rand(common)
            for n in own:
                self.lens.append(common + n)
                self.leader.append(first)
                self.shared.append(common)
                plan.append((torch.cat([k0, rand(n)]), torch.cat([v0, rand(n)])))
        need = [-(-n // page) for n in self.lens]
        order = torch.randperm(sum(need) + 1, generator=g).tolist()
        n_pages, width = len(order), max(need + [1]) + 2
        self.table_host = torch.full((len(need), width), n_pages + 7, dtype=torch.int32)
        fill = 127 if int8 else float("nan")
        pools = [torch.full((n_pages, n_kv, page, dim), fill, dtype=torch.int8 if int8 else torch.bfloat16) for _ in range(2)]
        self.scales = [(torch.rand(n_kv, generator=g) * 0.5 + 0.5) / 40 for _ in range(2)] if int8 else [None, None]
        self.k, self.v = [], []
        for b, rows in enumerate(plan):
            for e in range(need[b]):
                l = self.leader[b]
                whole = (e + 1) * page <= self.shared[b] and l != b
                self.table_host[b, e] = self.table_host[l, e] if whole else order.pop()
            for pool, x, out, scale in zip(pools, rows, (self.k, self.v), self.scales):
                y = (x * 40).round().clamp(-128, 127).to(torch.int8) if int8 else x.to(torch.bfloat16)
                for e in range(need[b]):
                    part = y[e * page:(e + 1) * page]
                    pool[self.table_host[b, e], :, :part.shape[0]] = part.transpose(0, 1)
                val = y.double()
                out.append((val * scale.double()[:, None] if int8 else val).numpy())
        if token_layout:
            pools = [p.permute(0, 2, 1, 3).contiguous().to(DEV).permute(0, 2, 1, 3) for p in pools]
        self.K, self.V = (p.to(DEV) for p in pools)
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
        self.table, self.kv_len = self.table_host.to(DEV), ints(self.lens)
        self.d_leader, self.d_shared = ints(self.leader), ints(self.shared)
        self.cache = B.KVCache(self.K, self.V, *(None if s is None else s.to(DEV) for s in self.scales))


def _queries(new, hq, dim, seed=1, scale=1.2):
    return (torch.randn((sum(new), hq * dim), generator=torch.Generator().manual_seed(seed)) * scale).to(torch.bfloat16)


def _run(pg, q, new, hq, perm=None, max_q=None, leader=None, shared=None, ws=None, lse=True, pad=0, ok=True):
    total, dim = sum(new), pg.dim
    wide = torch.zeros((total + 3, hq * dim + pad), dtype=torch.bfloat16, device=DEV)
    wide[:total, :hq * dim] = q.to(DEV)
    o_full, lse_full = torch.full((total + 3, hq * dim + pad), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((total + 3, hq), 7.0, device=DEV)
    max_q = max(new + [0]) if max_q is None else max_q
    if ws is None:
        ws = B.new_kv_attention_shared_workspace(len(new), total, max_q, pg.table.shape[1], hq, pg.cache)
        ws[256:] = 0xff                             # nothing of it is read before it is written
    dperm = None if perm is None else torch.tensor(np.concatenate(perm), dtype=torch.int32, device=DEV)
    B.mq_kv_attention_shared(wide[:total, :hq * dim], cu(new), pg.kv_len, pg.table, pg.d_leader if leader is None else leader,
                             pg.d_shared if shared is None else shared, pg.cache, hq, max_q, o_full[:total, :hq * dim], ws,
                             lse=lse_full[:total] if lse else None, perm=dperm)
    torch.cuda.synchronize()
    assert not ok or B.mq_last_device_status(ws) == (B.MQ_OK, 0)
    assert bool((o_full[total:] == 7.0).all()) and bool((lse_full[total:] == 7.0).all()) and bool((o_full[:, hq * dim:] == 7.0).all())
    return o_full[:total, :hq * dim].float().cpu().numpy().astype(np.float64), lse_full[:total].cpu().numpy().astype(np.float64)


def _check(pg, q, new, hq, o, lse, perm=None, heads=None, skip=()):
    group, dim = hq // pg.n_kv, pg.dim
    scale = dim ** -0.5
    qf = q.double().numpy().reshape(-1, hq, dim)
    p_step = 2.0 ** -11 if pg.int8 else 2.0 ** -8
    start = 0
    for b, n in enumerate(new):
        for h in (range(hq) if heads is None else heads):
            if b in skip:
                break
            g = h // group
            ref, ref_lse, _, abs_pv, mag = O.attention(qf[start:start + n, h], pg.k[b][:, g], pg.v[b][:, g], scale, None if perm is None else perm[b])
            got = o[start:start + n, h * dim:(h + 1) * dim]
            ds = (dim + 8) * 2.0 ** -23 * mag[:, None]
            tol = 2.0 ** -8 * np.abs(ref) + (p_step + 2 * ds + 2.0 ** -19 + 2.0 ** -20) * abs_pv + 1e-30
            if pg.int8:
                tol = tol + 2.0 ** -31 * np.abs(pg.v[b][:, g]).sum(0)
            assert np.all(np.abs(got - ref) <= tol), (b, h, float((np.abs(got - ref) / tol).max()))
            dead, got_l = np.isneginf(ref_lse), lse[start:start + n, h]
            assert np.array_equal(dead, np.isneginf(got_l))
            assert np.all(np.abs(got_l - ref_lse)[~dead] <= (ds[:, 0] + 2.0 ** -19 * (1 + np.abs(ref_lse)))[~dead])
        start += n


CASES = [
    # new tokens, groups (keys in common, keys of its own), hq, hkv, dim, page, int8, aifs
    ([1] * 4, [(128, [1, 5, 40, 17])], 8, 2, 128, 16, False, False),                      # 16 rows: the kernel for few rows on both lines
    ([1] * 12, [(640, [1, 2, 30, 64, 65, 100, 7, 8, 9, 10, 300, 1])], 28, 4, 128, 64, False, False),
    ([1] * 10, [(1000, [3] * 4), (90, [10, 11, 12]), (2000, [500, 1, 2])], 32, 8, 128, 32, False, False),   # groups of different length, a remainder
    ([1] * 9, [(500, [20, 33]), (0, [100]), (300, [1]), (256, [40, 1, 9]), (0, [5, 6])], 16, 2, 64, 16, False, False),
    ([1] * 20, [(700, list(range(1, 21)))], 14, 2, 128, 64, True, False),
    ([1] * 3, [(333, [1, 50, 130])], 4, 2, 64, 16, True, False),
    ([3, 1, 0, 2, 5], [(400, [3, 8, 0, 2, 90])], 28, 4, 128, 64, False, False),           # one sequence without rows, one whose rows are all of its own keys
    ([40, 7, 100, 33], [(512, [40, 60, 100, 200])], 8, 4, 128, 128, False, False),
    ([20, 35, 1, 18], [(300, [25, 80]), (96, [1, 60])], 14, 2, 64, 16, False, True),      # AIFS order behind the shared keys
    ([40, 90], [(256, [50, 100])], 8, 2, 128, 256, True, True),
    ([1, 1], [(70, [1, 1])], 2, 2, 128, 64, False, False),
    ([1] * 2, [(130, [9, 4])], 130, 1, 128, 16, False, False),                            # more query heads per key/value head than a block has rows
    ([2] * 150, [(200, [2 + i % 5 for i in range(150)])], 7, 1, 64, 16, False, False),    # several blocks of rows, none of whole sequences
    ([1] * 5, [(4000, [60, 1, 400, 2, 8])], 6, 1, 128, 64, False, False),                 # few rows spread over all workers
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_shared(case):
    new, groups, hq, hkv, dim, page, int8, aifs = CASES[case]
    pg = Groups(groups, hkv, dim, page, int8, token_layout=case % 2 == 1, seed=case)
    q = _queries(new, hq, dim, seed=50 + case)
    perm = aifs_perm(np.random.default_rng(case), new) if aifs else None
    o, lse = _run(pg, q, new, hq, perm, pad=24 if case % 3 == 0 else 0)
    _check(pg, q, new, hq, o, lse, perm, heads=None if hq <= 8 else sorted({0, hq // hkv - 1, hq - 1, hq // 2}))


def test_shared_lengths_are_bounds():
    """More than a sequence has in front of its rows, or less than it could be; loose host bounds; no log-sum-exps."""
    new, groups = [1, 2, 1, 1], [(200, [1, 30, 5, 77])]
    pg = Groups(groups, 2, 128, 16, seed=3)
    q = _queries(new, 8, 128)
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)
    first = _run(pg, q, new, 8)
    for shared in (ints(200, 200, 200, 200), ints(100, 200, 200, 200), ints(0, 200, 200, 200), ints(15, 300, 16, -4), ints(200, 207, 200, 205)):
        _check(pg, q, new, 8, *_run(pg, q, new, 8, shared=shared))
    _check(pg, q, new, 8, *_run(pg, q, new, 8, max_q=5))
    assert np.array_equal(_run(pg, q, new, 8, lse=False)[0], first[0])
    # what the sequences have in common by themselves bounds it where shared_len says more than their contexts hold
    pg = Groups([(192, [1, 1, 40])], 2, 128, 16, seed=4)
    q = _queries([1, 1, 1], 8, 128)
    _check(pg, q, [1, 1, 1], 8, *_run(pg, q, [1, 1, 1], 8, shared=ints(1 << 30, 1 << 30, 192)))


def test_leaders_that_say_nothing_of_use():
    """Not side by side, behind the sequence, chains, numbers out of range: every sequence reads by itself."""
    new, groups = [1, 1, 1, 1, 1], [(160, [1, 30, 5, 77, 8])]
    pg = Groups(groups, 2, 64, 16, seed=5)
    q = _queries(new, 4, 64)
    for leader in ([0, 1, 0, 1, 0], [0, 0, 1, 1, 3], [4, 4, 4, 4, 4], [-1, 9, 1 << 30, -7, 4], [1, 1, 1, 3, 3], [0, 1, 2, 3, 4], [0, 0, 2, 2, 0]):
        _check(pg, q, new, 4, *_run(pg, q, new, 4, leader=torch.tensor(leader, dtype=torch.int32, device=DEV)))


def test_rows_that_belong_to_no_sequence_or_see_nothing():
    pg = Groups([(96, [4, 1, 3])], 2, 64, 16, seed=6)
    q = _queries([2, 1, 2], 4, 64)
    ws = B.new_kv_attention_shared_workspace(3, 5, 2, pg.table.shape[1], 4, pg.cache)
    for cu_q, live in (([0, 1, 2, 4], [0, 1, 2, 3]), ([1, 2, 3, 5], [1, 2, 3, 4]), ([0, 0, 0, 0], [])):
        o, lse = torch.full((5, 256), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((5, 4), 7.0, device=DEV)
        B.mq_kv_attention_shared(q.to(DEV), torch.tensor(cu_q, dtype=torch.int32, device=DEV), pg.kv_len, pg.table, pg.d_leader, pg.d_shared, pg.cache,
                                 4, 2, o, ws, lse=lse)
        torch.cuda.synchronize()
        dead = [i for i in range(5) if i not in live]
        assert bool((o[dead] == 7.0).all()) and bool((lse[dead] == 7.0).all()) and bool((o[live] != 7.0).any(1).all())
    short = Groups([(96, [4, 1, 3])], 2, 64, 16, seed=6)          # fewer keys than rows: some rows see nothing
    short.lens = [100, 97, 1]
    short.kv_len[2] = 1
    short.k[2], short.v[2] = short.k[2][:1], short.v[2][:1]
    o, lse = _run(short, q, [2, 1, 2], 4)
    _check(short, q, [2, 1, 2], 4, o, lse)


@pytest.mark.parametrize("n", [3, 40])
@pytest.mark.parametrize("int8", [False, True])
def test_bad_pages_read_as_zeros_and_are_reported(n, int8):
    pg = Groups([(320, [20 + i for i in range(n)])], 1, 128, 64, int8, seed=7)
    q = _queries([1] * n, 4, 128)
    pg.table[0, 1] = pg.K.shape[0] + 3                                # a shared page, of all sequences
    for b in range(n):
        pg.k[b][64:128] = 0.0
        pg.v[b][64:128] = 0.0
    ws = B.new_kv_attention_shared_workspace(n, n, 1, pg.table.shape[1], 4, pg.cache)
    o, lse = _run(pg, q, [1] * n, 4, ws=ws, ok=False)
    assert B.mq_last_device_status(ws)[0] == B.MQ_ERR_INVALID_ARG
    _check(pg, q, [1] * n, 4, o, lse)


def test_infinite_and_nan_values_reach_those_who_see_them():
    """A shared value reaches every row, one of a sequence's own only its rows, one of a later row nobody before it."""
    new = [2, 1, 2]
    for n_more in (0, 30):                                             # few rows, and enough for the other kernel
        groups = [(128, [5, 9, 40] + [1] * n_more)]
        news = new + [1] * n_more
        pg = Groups(groups, 1, 64, 16, seed=8)
        q = _queries(news, 4, 64)
        last = pg.lens[0] - 1                                          # seen by the second row of sequence 0 only
        pg.V[pg.table_host[0, last // 16].item(), 0, last % 16, 3] = float("nan")
        own = 130                                                      # of sequence 2
        pg.V[pg.table_host[2, own // 16].item(), 0, own % 16, 5] = float("inf")
        o, _ = _run(pg, q, news, 4)
        bad = ~np.isfinite(o.reshape(-1, 4, 64))
        want = np.zeros_like(bad)
        want[1, :, 3] = True
        want[3:5, :, 5] = True
        assert np.array_equal(bad, want)
        pg.V[pg.table_host[0, 2].item(), 0, 7, 9] = float("inf")      # key 39, shared
        o, _ = _run(pg, q, news, 4)
        want[:, :, 9] = True
        assert np.array_equal(~np.isfinite(o.reshape(-1, 4, 64)), want)


def test_equal_to_the_plain_call_and_the_same_every_time():
    new = [1] * 24
    pg = Groups([(1500, [i * 7 + 1 for i in range(24)])], 4, 128, 32, seed=9)
    q = _queries(new, 28, 128)
    a = _run(pg, q, new, 28)
    for _ in range(3):
        b = _run(pg, q, new, 28)
        assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])
    ws = B.new_kv_attention_workspace(24, 24, 1, pg.table.shape[1], 28, pg.cache)
    o = torch.empty((24, 28 * 128), dtype=torch.bfloat16, device=DEV)
    B.mq_kv_attention(q.to(DEV), cu(new), pg.kv_len, pg.table, pg.cache, 28, 1, o, ws)
    plain = o.double().cpu().numpy()
    scale = np.abs(plain).max()                                        # each is within its tolerance of the same numbers
    assert np.abs(plain - a[0]).max() <= 4 * 2.0 ** -8 * max(1.0, scale) * 2


def test_captured_graph_follows_groups_and_lengths():
    a, b = Groups([(600, [9, 30, 1, 4]), (64, [2, 3])], 2, 128, 16, seed=10), Groups([(48, [3, 5]), (320, [40, 1, 9, 200])], 2, 128, 16, seed=11)
    new = [1] * 6
    width = max(a.table.shape[1], b.table.shape[1])
    pages = max(a.K.shape[0], b.K.shape[0])
    K, V = (torch.zeros((pages, 2, 16, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    table = torch.zeros((6, width), dtype=torch.int32, device=DEV)
    q, o = torch.zeros((6, 1024), dtype=torch.bfloat16, device=DEV), torch.zeros((6, 1024), dtype=torch.bfloat16, device=DEV)
    lse = torch.zeros((6, 8), device=DEV)
    kv, leader, shared = (torch.zeros(6, dtype=torch.int32, device=DEV) for _ in range(3))
    cache = B.KVCache(K, V)
    ws = B.new_kv_attention_shared_workspace(6, 6, 1, width, 8, cache)
    c = cu(new)
    call = lambda: B.mq_kv_attention_shared(q, c, kv, table, leader, shared, cache, 8, 1, o, ws, lse=lse)
    kv.fill_(1)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for pg in (a, b, a):
        K[:pg.K.shape[0]], V[:pg.V.shape[0]] = pg.K, pg.V
        table[:, :pg.table.shape[1]] = pg.table
        kv.copy_(pg.kv_len), leader.copy_(pg.d_leader), shared.copy_(pg.d_shared)
        hq = _queries(new, 8, 128, seed=12)
        q.copy_(hq)
        graph.replay()
        torch.cuda.synchronize()
        assert B.mq_last_device_status(ws) == (B.MQ_OK, 0)
        _check(pg, hq, new, 8, o.double().cpu().numpy(), lse.double().cpu().numpy())


def test_the_most_sequences_and_empty_calls():
    n = 1024
    pg = Groups([(32, [1 + i % 3 for i in range(n)])], 1, 64, 16, seed=13)
    q = _queries([1] * n, 2, 64)
    o, lse = _run(pg, q, [1] * n, 2)
    _check(pg, q, [1] * n, 2, o, lse)
    q40 = _queries([40] + [1] * (n - 1), 2, 64)
    pg = Groups([(32, [40] + [1 + i % 3 for i in range(n - 1)])], 1, 64, 16, True, seed=14)
    o, lse = _run(pg, q40, [40] + [1] * (n - 1), 2)
    _check(pg, q40, [40] + [1] * (n - 1), 2, o, lse)
    ws = torch.zeros(1 << 16, dtype=torch.uint8, device=DEV)
    empty = torch.empty((0, 128), dtype=torch.bfloat16, device=DEV)
    B.mq_kv_attention_shared(empty, cu([0] * n), pg.kv_len, pg.table, pg.d_leader, pg.d_shared, pg.cache, 2, 0, empty, ws)


def test_two_streams_with_their_own_workspaces():
    pgs = [Groups([(900, [5, 60, 200, 1])], 2, 128, 32, seed=s) for s in (15, 16)]
    qs = [_queries([1] * 4, 8, 128, seed=s) for s in (1, 2)]
    want = [_run(pg, q, [1] * 4, 8) for pg, q in zip(pgs, qs)]
    c = cu([1] * 4)
    bufs = [(q.to(DEV), torch.empty((4, 1024), dtype=torch.bfloat16, device=DEV),
             B.new_kv_attention_shared_workspace(4, 4, 1, pg.table.shape[1], 8, pg.cache)) for pg, q in zip(pgs, qs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        for st, pg, (q, o, ws) in zip(streams, pgs, bufs):
            with torch.cuda.stream(st):
                B.mq_kv_attention_shared(q, c, pg.kv_len, pg.table, pg.d_leader, pg.d_shared, pg.cache, 8, 1, o, ws)
    torch.cuda.synchronize()
    for (_, o, _), (w, _) in zip(bufs, want):
        assert np.array_equal(o.double().cpu().numpy(), w)


@pytest.mark.parametrize("n_heads", [2, 16])
def test_row_counts_that_decrease_share_nothing(n_heads):
    """A cu_q that is not one: every sequence reads by itself what mq_kv_attention reads for it, and the call ends as soon."""
    pg = Groups([(160, [1, 30, 5, 77, 8])], 2, 64, 16, seed=17)
    dev = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
    for rows, cu_q in ((12, [10, 12, 2, 4, 4, 7]), (12, [8, 9, 6, 7, 2, 3]), (12, [12, 0, 0, 1, 1, 1]), (12, [5, 6, 6, 7, 8, 3]),
                       (12, [900, -4, 2, 3, 1 << 30, 11]), (12, [0, 6, 10, 3, 4, 5]), (700, [690, 692, 2, 4, 4, 7]), (700, [699, 0, 600, 601, 100, 102])):
        q = _queries([rows], n_heads, 64, seed=18).to(DEV)
        ws = B.new_kv_attention_workspace(5, rows, 2, pg.table.shape[1], n_heads, pg.cache)
        wss = B.new_kv_attention_shared_workspace(5, rows, 2, pg.table.shape[1], n_heads, pg.cache)
        a, b = (torch.full((rows, n_heads * 64), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        B.mq_kv_attention(q, dev(cu_q), pg.kv_len, pg.table, pg.cache, n_heads, 2, a, ws)
        B.mq_kv_attention_shared(q, dev(cu_q), pg.kv_len, pg.table, pg.d_leader, pg.d_shared, pg.cache, n_heads, 2, b, wss)
        torch.cuda.synchronize()
        assert B.mq_last_device_status(wss) == B.mq_last_device_status(ws) == (B.MQ_OK, 0)
        begin = [min(max(c, 0), rows) for c in cu_q[:-1]]
        spans = [(lo, min(min(max(hi, lo), rows) - lo, 2)) for lo, hi in zip(begin, cu_q[1:])]
        owned = [sum(lo <= r < lo + n for lo, n in spans) for r in range(rows)]
        assert max(owned) == 1
        most = float(pg.V[pg.V == pg.V].abs().max())         # of a value, and so of a result and of the sums of absolute values
        for r in range(rows):
            if owned[r]:                                     # (each within two roundings to bf16 and a probability's, besides float32 sums)
                assert float((a[r].float() - b[r].float()).abs().max()) <= 2 * (2.0 ** -8 + 2.0 ** -8 + 2.0 ** -10) * most, (cu_q, r)
            else:
                assert bool((a[r] == 7.0).all()) and bool((b[r] == 7.0).all())
