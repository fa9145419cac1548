"""mq_kv_plan against the definition: whole numbers, equal throughout."""
import copy

import numpy as np
import pytest
import torch

from oracle.plan_oracle import Refused, plan
from paper_2502_00425_b200 import binding as B

from kv_util import DEV

pytestmark = pytest.mark.gpu


class Pool:
    """The same state on the host (lists) and on the GPU."""

    def __init__(self, lens, width, n_pages, page, borrowed=None, seed=0):
        rng = np.random.default_rng(seed)
        order = rng.permutation(n_pages).tolist()
        n = len(lens)
        table, lent = [[-7] * width for _ in lens], borrowed or [0] * n
        for b, l in enumerate(lens):
            for e in range(-(-l // page)):
                table[b][e] = 10 ** 6 + e if e < lent[b] else order.pop()   # (a borrowed page must not turn up in the free list)
        self.page = page
        self.host = dict(kv_len=list(lens), seen=[l + 3 * b if l else 0 for b, l in enumerate(lens)], borrowed=list(lent), table=table,
                         free=order, n_pages=n_pages)
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
        free = ints(order + [-9] * (n_pages - len(order)))
        self.dev = dict(kv_len=ints(self.host["kv_len"]), seen=ints(self.host["seen"]), table=ints(table).view(n, width), free=free,
                        n_free=ints([len(order)]), borrowed=ints(lent) if borrowed else None)
        d = self.dev
        self.state = B.KVState(d["kv_len"], d["seen"], d["table"], d["free"], d["n_free"], page, borrowed=d["borrowed"])
        self.status = torch.zeros(2, dtype=torch.int32, device=DEV)

    def step(self, new, keep=None, max_rows=None):
        rows = sum(new) if max_rows is None else max_rows
        n = len(new)
        ints = lambda v: None if v is None else torch.tensor(v, dtype=torch.int32, device=DEV)
        cu = torch.full((n + 2,), 99, dtype=torch.int32, device=DEV)
        slots, pos = torch.full((rows + 1,), 99, dtype=torch.int64, device=DEV), torch.full((rows + 1,), 99, dtype=torch.int32, device=DEV)
        before = {k: None if v is None else v.clone() for k, v in self.dev.items()}
        self.status.zero_()
        B.mq_kv_plan(self.state, ints(new), cu[:n + 1], slots[:rows], pos[:rows], self.status, keep=ints(keep))
        torch.cuda.synchronize()
        assert cu[n + 1] == 99 and slots[rows] == 99 and pos[rows] == 99
        try:
            want = plan(self.host, new, keep, rows, self.page)
        except Refused as e:
            assert self.status.tolist() == [B.MQ_ERR_WORKSPACE if e.args[0] == 4 else B.MQ_ERR_INVALID_ARG, e.args[0]]
            assert bool((cu[:n + 1] == 0).all()) and bool((slots[:rows] == -1).all()) and bool((pos[:rows] == 0).all())
            assert all(v is None or torch.equal(v, self.dev[k]) for k, v in before.items())
            return None
        assert self.status.tolist() == [0, 0]
        assert (cu[:n + 1].tolist(), slots[:rows].tolist(), pos[:rows].tolist()) == want
        self.check()
        return want

    def check(self):
        h, d = self.host, self.dev
        assert d["kv_len"].tolist() == h["kv_len"] and d["seen"].tolist() == h["seen"] and d["table"].tolist() == h["table"]
        assert int(d["n_free"]) == len(h["free"]) and d["free"][:len(h["free"])].tolist() == h["free"]
        if d["borrowed"] is not None:
            assert d["borrowed"].tolist() == h["borrowed"]


@pytest.mark.parametrize("n_seq,page,seed", [(1, 16, 0), (3, 64, 1), (40, 16, 2), (257, 32, 3), (1024, 128, 4), (1025, 16, 5), (2048, 256, 6)])
def test_random_steps(n_seq, page, seed):
    """Growth by nothing, one token and many, cuts, ends and new beginnings, and steps that cannot be made among them."""
    rng = np.random.default_rng(seed)
    width = 12 if n_seq > 300 else 40
    lens = rng.integers(0, width * page // 2, n_seq).tolist()
    pool = Pool(lens, width, n_seq * width // 2 + 5, page, seed=seed)
    made = 0
    for i in range(8):
        kind = rng.integers(0, 4, n_seq)
        new = np.where(kind == 0, 0, np.where(kind < 3, rng.integers(1, 3, n_seq), rng.integers(0, width * page // 8, n_seq))).tolist()
        keep = [int(rng.integers(0, l + 5)) if c < 0.3 else 0 if c < 0.4 else 1 << 30 for l, c in zip(pool.host["kv_len"], rng.random(n_seq))]
        made += pool.step(new, keep if i % 2 else None, max_rows=sum(new) + int(rng.integers(0, 40))) is not None
    assert made >= 4


def test_a_step_is_taken_back():
    rng = np.random.default_rng(9)
    pool = Pool(rng.integers(0, 300, 60).tolist(), 40, 1500, 16, seed=9)
    for _ in range(4):
        before = copy.deepcopy(pool.host)
        new = rng.integers(0, 90, 60).tolist()
        assert pool.step(new)
        assert pool.step([0] * 60, keep=before["kv_len"], max_rows=0)
        assert {k: pool.host[k] for k in ("kv_len", "free")} == {k: before[k] for k in ("kv_len", "free")}
        assert pool.host["seen"] == [s if l else 0 for s, l in zip(before["seen"], before["kv_len"])]
        pool.step(rng.integers(0, 5, 60).tolist())


def test_borrowed_pages():
    page = 16
    pool = Pool([100, 64, 40, 48, 0], 10, 30, page, borrowed=[2, 4, 0, 1, 0], seed=1)
    assert pool.step([1, 1, 1, 1, 1])
    assert pool.step([0, 0, 0, 0, 3], keep=[32, 64, 40, 16, 0])          # cut down to what is borrowed
    assert pool.step([5, 20, 0, 33, 0])
    assert pool.step([40, 0, 0, 0, 0], keep=[16, 48, 40, 0, 3])          # inside it, at whole pages: the rest is its own anew
    assert pool.host["borrowed"] == [1, 3, 0, 0, 0]
    assert pool.step([0] * 5, keep=[8, 48, 40, 0, 3]) is None            # not inside a page
    assert pool.step([0] * 5, keep=[0] * 5)
    assert len(pool.host["free"]) == 30 - 0 and pool.host["borrowed"] == [0] * 5
    pool.dev["borrowed"][1] = 1                                           # more than it has keys
    pool.host["borrowed"][1] = 1
    assert pool.step([0] * 5) is None


def test_what_cannot_be_done():
    pool = Pool([30, 0, 16], 4, 8, 16)
    assert pool.step([1, -1, 0], max_rows=10) is None
    assert pool.step([35, 0, 0]) is None                                  # behind the table's reach
    assert pool.step([1, 1, 1], keep=[30, 0, -1]) is None
    assert pool.step([5, 5, 5], max_rows=14) is None
    assert pool.step([30, 40, 40]) is None                                # 2 + 3 + 3 pages, five are free
    assert pool.step([2, 60, 16]) is not None                             # all five
    assert pool.step([0, 1, 1]) is None
    assert pool.step([0, 5, 20], keep=[0, 60, 20]) is None and pool.step([0, 4, 20], keep=[0, 60, 12]) is not None
    pool.dev["n_free"].fill_(7)                                           # a list that says too much
    pool.host["free"] = pool.host["free"] + [1] * (7 - len(pool.host["free"]))
    assert pool.step([0, 0, 0], keep=[0, 0, 0]) is None
    pool.dev["kv_len"][0] = 1 << 20
    pool.host["kv_len"][0] = 1 << 20
    assert pool.step([0, 0, 0]) is None


def test_many_rows_and_long_rows():
    """More than one block places, and one sequence has thousands of pages."""
    pool = Pool([0, 70000, 17], 9000, 20000, 16)
    assert pool.step([131, 70000, 4000], max_rows=80000)
    assert pool.step([0, 0, 0], keep=[0, 5, 0], max_rows=4097)
    assert pool.step([100000, 0, 0])
    Pool([0] * 2048, 3, 5000, 16).step([2] * 2048, max_rows=4096)
    Pool([0] * 2048, 3, 5000, 16).step([2] * 2048, max_rows=4097)


def test_no_sequences():
    pool = Pool([], 0, 4, 16)
    assert pool.step([], max_rows=3) == ([0], [-1] * 3, [0] * 3)


def test_captured_steps_follow_the_state():
    pool = Pool([10, 20, 0, 31], 30, 100, 16)
    new = torch.tensor([1, 1, 0, 1], dtype=torch.int32, device=DEV)
    cu = torch.zeros(5, dtype=torch.int32, device=DEV)
    slots, pos = torch.zeros(6, dtype=torch.int64, device=DEV), torch.zeros(6, dtype=torch.int32, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.mq_kv_plan(pool.state, new, cu, slots, pos, pool.status)
    for i in range(40):
        if i == 20:
            new.copy_(torch.tensor([0, 2, 3, 1], device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        want = plan(pool.host, new.tolist(), None, 6, 16)
        assert (cu.tolist(), slots.tolist(), pos.tolist()) == want
        pool.check()
