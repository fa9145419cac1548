"""mq_sample against the float64 definition.

Tokens and counts have to be equal: a weight of the call is off by at most 2^-44 of the largest one and 2^-37 of itself (fixed point; a table
and a cubic in double), so a border (top_p, u) lies within 2^-36 of its place relative to the total, plus V 2^-44 of the largest weight in the worst
case.  A random border comes that near to a token's edge once in 2^36 / tokens rows (some 2^19 rows for 10^5 tokens); the constructed
cases sum exactly.  logp is one float32 rounding (2^-24, relative) of a logarithm whose argument is off by 2^-30 at most.
"""
import numpy as np
import pytest
import torch

from oracle.sample_oracle import sample
from paper_2502_00425_b200 import binding as B

from kv_util import DEV

pytestmark = pytest.mark.gpu


def _run(x, t, u, k=None, p=None, mp=None):
    n = x.shape[0]
    dev = lambda v, dt: None if v is None else torch.tensor(np.broadcast_to(np.asarray(v), (n,)).copy(), dtype=dt, device=DEV)
    token, kept = (torch.full((n + 1,), 77, dtype=torch.int32, device=DEV) for _ in range(2))
    logp = torch.full((n + 1,), 77.0, device=DEV)
    B.mq_sample(x, dev(t, torch.float32), dev(u, torch.float32), token[:n], top_k=dev(k, torch.int32), top_p=dev(p, torch.float32),
                min_p=dev(mp, torch.float32), logp=logp[:n], kept=kept[:n])
    torch.cuda.synchronize()
    assert int(token[n]) == 77 and float(logp[n]) == 77.0 and int(kept[n]) == 77
    return token[:n].tolist(), logp[:n].double().tolist(), kept[:n].tolist()


def _check(x, t, u, k=None, p=None, mp=None):
    got = _run(x, t, u, k, p, mp)
    host = x.float().cpu().numpy()
    at = lambda v, r, off: off if v is None else np.broadcast_to(np.asarray(v), (x.shape[0],))[r]
    for r, (token, logp, kept) in enumerate(zip(*got)):
        want, lp, keep = sample(host[r], at(t, r, 0), at(u, r, 0), at(k, r, 0), at(p, r, 1.0), at(mp, r, 0.0))
        assert (token, kept) == (want, keep.size), (r, token, kept, want, keep.size)
        assert logp == lp or abs(logp - lp) <= 2.0 ** -24 * abs(lp) + 2.0 ** -30, (r, logp, lp)
    return got


def _logits(rng, n, v, bf16, peaks=40):
    x = rng.standard_normal((n, v)) * 2
    for r in range(n):
        at = rng.integers(0, v, min(v, peaks))
        x[r, at] += 8 + 3 * rng.standard_normal(at.size)
    t = torch.from_numpy(x.astype(np.float32))
    return (t.to(torch.bfloat16) if bf16 else t).to(DEV)


@pytest.mark.parametrize("v", [1, 2, 7, 33, 1000, 4095, 4096, 9999, 20001, 131072])
@pytest.mark.parametrize("bf16", [False, True])
def test_every_filter(v, bf16):
    rng = np.random.default_rng(v)
    n = 24
    x = _logits(rng, n, v, bf16)
    t = rng.uniform(0.4, 1.6, n).astype(np.float32)
    u = rng.random(n).astype(np.float32)
    k = np.where(np.arange(n) % 3 == 0, rng.integers(1, v + 2, n), rng.integers(1, 60, n))
    p, mp = rng.uniform(0.1, 0.98, n).astype(np.float32), rng.uniform(1e-4, 0.3, n).astype(np.float32)
    _check(x, t, u)
    _check(x, t, u, k=k)
    _check(x, t, u, p=p)
    _check(x, t, u, mp=mp)
    _check(x, t, u, k=k, p=p, mp=mp)
    _check(x, np.where(np.arange(n) % 2, 0.0, t), u, k=np.where(np.arange(n) % 4 < 2, k, 0), p=np.where(np.arange(n) % 5 < 3, p, 1.0), mp=mp)


@pytest.mark.parametrize("bf16", [False, True])
def test_flat_rows(bf16):
    """Thousands of tokens are kept: nothing fits into a list."""
    rng = np.random.default_rng(1)
    n, v = 8, 100003
    x = (torch.from_numpy(rng.standard_normal((n, v)).astype(np.float32) * 0.5).to(torch.bfloat16 if bf16 else torch.float32)).to(DEV)
    u = rng.random(n).astype(np.float32)
    for kw in (dict(), dict(p=0.9), dict(p=0.5), dict(k=30000), dict(k=30000, p=0.95), dict(k=50000, p=0.3, mp=0.2), dict(mp=0.1)):
        _check(x, 1.0, u, **kw)
    _check(x, 30.0, u, k=20000)        # a temperature that makes it flatter still
    _check(x, 0.02, u, p=0.9)          # and ones that leave few
    _check(x, 0.0005, u, k=500)


@pytest.mark.parametrize("v", [5000, 60000])
def test_equal_logits_are_cut_by_index(v):
    x = torch.full((4, v), 1.5, device=DEV)
    u = np.array([0.0, 0.25, 0.5, 0.99999994], np.float32)
    tok, _, kept = _check(x, 0.7, u)
    assert tok[0] == 0 and tok[2] == v // 2 and tok[3] == v - 1 and kept == [v] * 4
    tok, _, kept = _check(x, 0.7, u, k=v - 3)
    assert kept == [v - 3] * 4 and max(tok) < v - 3
    _, _, kept = _check(x, 0.7, u, p=0.5)
    assert kept == [v // 2] * 4
    _, _, kept = _check(x, 0.7, u, p=0.25, k=4 * (v // 8))
    assert kept == [v // 8] * 4
    _check(x, 0.7, u, mp=1.0)
    y = x.clone()                      # two values, the larger at every third column
    y[:, ::3] = 2.5
    n3 = -(-v // 3)
    for k in (n3 - 1, n3, n3 + 1, n3 + 1000, v - 1):
        _check(y, 1.0, u, k=k)
    _check(y, 1.0, u, p=0.9)
    _check(y, 0.5, u, p=0.2, k=n3 + 7)
    z = y.clone()
    z[:, 1::3] = -0.0
    z[:, 2::3] = 0.0                   # one value, two bit patterns
    _check(z, 1.0, u, k=n3 + 501)


def test_masked_rows_nans_and_infinities():
    rng = np.random.default_rng(2)
    v, inf, nan = 30011, float("inf"), float("nan")
    x = _logits(rng, 10, v, False)
    x[0] = -inf
    x[1] = nan
    x[2, 100:] = -inf
    x[3, :-1] = nan
    x[4, ::2] = -inf
    x[5, 77] = inf
    x[6, 5:2000:7] = inf
    x[7, 1000:20000] = torch.finfo(torch.float32).min
    x[8] = torch.finfo(torch.float32).min
    x[9, :] = -inf
    x[9, 12345] = torch.finfo(torch.float32).min
    u = rng.random(10).astype(np.float32)
    for kw in (dict(), dict(k=200), dict(k=5000), dict(p=0.8), dict(mp=0.05), dict(k=20000, p=0.9, mp=0.001)):
        tok, lp, kept = _check(x, 0.9, u, **kw)
        assert tok[:2] == [-1, -1] and kept[:2] == [0, 0] and lp[0] == -np.inf and tok[3] == v - 1 and tok[5] == 77 and tok[9] == 12345
    tok, _, _ = _check(x, 0.0, u)
    assert tok[0] == -1 and tok[5] == 77 and tok[6] == 5 and tok[8] == 0
    w = x.to(torch.bfloat16)
    _check(w, 0.9, u, p=0.8, k=7000)


def test_extreme_parameters():
    rng = np.random.default_rng(3)
    n, v = 6, 12000
    x = _logits(rng, n, v, False)
    u = rng.random(n).astype(np.float32)
    nan, inf = float("nan"), float("inf")
    for t in (nan, -1.0, 0.0):
        tok, lp, kept = _check(x, t, u, k=5)
        assert tok == x.argmax(1).tolist() and lp == [0.0] * n and kept == [1] * n
    _check(x, 1e-30, u, p=0.9)
    _check(x, 1e-42, u, k=300)
    tok, _, kept = _check(x, inf, u)
    assert kept == [v] * n and tok == [int(np.float64(a) * v) for a in u]      # every token alike
    _check(x, inf, u, k=5000)
    base = _run(x, 1.0, u)
    for kw in (dict(k=0), dict(k=-3), dict(k=v), dict(k=v + 5), dict(p=1.0), dict(p=1.5), dict(p=nan), dict(mp=0.0), dict(mp=-1.0), dict(mp=nan)):
        assert _run(x, 1.0, u, **kw) == base
    for kw in (dict(p=0.0), dict(p=-1.0), dict(p=1e-30), dict(k=1), dict(mp=5.0)):
        tok, _, kept = _run(x, 1.0, u, **kw)
        assert tok == x.argmax(1).tolist() and kept == [1] * n
    low, high = _run(x, 1.0, np.zeros(n, np.float32))[0], _run(x, 1.0, np.full(n, 0.99999994, np.float32))[0]
    assert _run(x, 1.0, np.full(n, -2.0))[0] == _run(x, 1.0, np.full(n, nan))[0] == low and _run(x, 1.0, np.full(n, 7.0))[0] == high


@pytest.mark.parametrize("bf16", [False, True])
def test_strides_and_offsets(bf16):
    """Rows that start anywhere in a 16-byte piece, poison around them."""
    rng = np.random.default_rng(4)
    v, dt = 10007, torch.bfloat16 if bf16 else torch.float32
    for pad, off in ((0, 0), (1, 0), (1, 1), (5, 3), (24, 7)):
        buf = torch.full((5, v + pad + off), float("inf"), dtype=dt, device=DEV)
        x = buf[:, off:off + v]
        x.copy_(_logits(rng, 5, v, bf16))
        _check(x, 0.8, rng.random(5).astype(np.float32), k=300, p=0.9)
        _check(x, 0.8, rng.random(5).astype(np.float32))
    _check(buf[2:3, off:off + v], 0.8, np.float32([0.3]), p=0.9)


def test_rows_too_long_to_be_staged():
    rng = np.random.default_rng(5)
    x = _logits(rng, 2, 1 << 19, False)
    u = rng.random(2).astype(np.float32)
    for kw in (dict(), dict(k=50), dict(p=0.9), dict(k=100000, p=0.99)):
        _check(x, 0.8, u, **kw)
    y = _logits(rng, 1, (1 << 20) - 5, True)
    _check(y, 1.0, u[:1], p=0.9, k=1000)


def test_sorted_rows():
    v = 40000
    x = torch.stack([torch.linspace(-20, 20, v), torch.linspace(20, -20, v), torch.linspace(-1e4, 1e4, v), torch.linspace(3e38, -3e38, v)]).to(DEV)
    u = np.array([0.1, 0.6, 0.9, 0.3], np.float32)
    for kw in (dict(), dict(k=64), dict(k=9000), dict(p=0.95), dict(k=9000, p=0.5), dict(mp=0.01)):
        _check(x, 1.0, u, **kw)


def test_captured_and_on_another_stream():
    rng = np.random.default_rng(6)
    n, v = 5, 9000
    x = torch.empty((n, v), device=DEV)
    t, u = torch.full((n,), 0.9, device=DEV), torch.empty(n, device=DEV)
    token = torch.empty(n, dtype=torch.int32, device=DEV)
    p = torch.full((n,), 0.9, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.mq_sample(x.zero_(), t, u.zero_(), token, top_p=p)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.mq_sample(x, t, u, token, top_p=p)
    for _ in range(3):
        x.copy_(_logits(rng, n, v, False))
        u.copy_(torch.from_numpy(rng.random(n).astype(np.float32)))
        graph.replay()
        torch.cuda.synchronize()
        host = x.cpu().numpy()
        assert token.tolist() == [sample(host[r], 0.9, float(u[r]), top_p=0.9)[0] for r in range(n)]


def test_no_rows_and_many_rows():
    _run(torch.empty((0, 100), device=DEV), 1.0, 0.5)
    rng = np.random.default_rng(7)
    x = _logits(rng, 700, 300, True, peaks=5)
    _check(x, 0.9, rng.random(700).astype(np.float32), k=20, p=0.9)


def test_the_drawn_tokens_have_their_probabilities():
    """20000 even steps of u: each token's share is its probability to one step."""
    v, n = 50, 20000
    x = torch.linspace(-3, 3, v, device=DEV).roll(13)
    tok, _, _ = _run(x.expand(n, v).contiguous(), 1.0, (np.arange(n) / n).astype(np.float32))
    prob = torch.softmax(x.double(), 0).cpu().numpy()
    share = np.bincount(tok, minlength=v) / n
    assert np.all(np.abs(share - prob) <= 1.0 / n + 2.0 ** -23)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("t", [0.03, 0.2, 1.0, 4.0])
def test_logits_that_crowd_in_a_corner_of_their_interval(bf16, t):
    """The mass of 1/32 wide intervals is first guessed from how many logits they have: here they lie at an end of theirs, or in a few of them."""
    rng = np.random.default_rng(int(100 * t))
    n, v = 6, 60013
    x = rng.standard_normal((n, v)) * np.array([0.3, 1.0, 2.0, 3.0, 0.1, 1.5])[:, None]
    low = np.floor(x * 32) / 32
    x = np.where(np.arange(n)[:, None] % 3 == 0, low + 1 / 33, np.where(np.arange(n)[:, None] % 3 == 1, low + 1e-4 * rng.random((n, v)), x))
    x[2] = np.round(x[2])
    x[5] -= 40.0
    x = torch.from_numpy(x.astype(np.float32))
    x = (x.to(torch.bfloat16) if bf16 else x).to(DEV)
    u, p = rng.random(n).astype(np.float32), rng.uniform(0.3, 0.97, n).astype(np.float32)
    k = rng.integers(3000, v, n)
    for kw in (dict(p=p), dict(p=p, k=k), dict(p=p, mp=0.3), dict(p=p, k=k, mp=0.02), dict(k=k)):
        _check(x, t, u, **kw)
    _check(x, t, np.float32(0.99999994), p=0.99, k=v - 1)


@pytest.mark.parametrize("bf16", [False, True])
def test_many_short_rows(bf16):
    rng = np.random.default_rng(11)
    n, v = 6000, 37
    x = _logits(rng, n, v, bf16, peaks=4)
    u, t = rng.random(n).astype(np.float32), rng.uniform(0.3, 2.0, n).astype(np.float32)
    _check(x, t, u, k=rng.integers(0, 50, n), p=rng.uniform(0.2, 1.2, n).astype(np.float32), mp=rng.uniform(-0.1, 0.2, n).astype(np.float32))


def test_rows_further_apart_than_32_bits():
    rng = np.random.default_rng(12)
    v, pitch = 20011, (1 << 31) + 8
    buf = torch.empty(2 * pitch + v, dtype=torch.bfloat16, device=DEV)
    x = buf.as_strided((3, v), (pitch, 1))
    x.copy_(_logits(rng, 3, v, True))
    _check(x, 0.8, rng.random(3).astype(np.float32), k=4000, p=0.9)
    del x, buf
    torch.cuda.empty_cache()


def test_two_calls_at_once():
    rng = np.random.default_rng(13)
    n, v = 40, 50021
    x, y = _logits(rng, n, v, False), (torch.from_numpy(rng.standard_normal((n, v)).astype(np.float32)) * 0.5).to(DEV)
    t, u, p = (torch.full((n,), f, device=DEV) for f in (0.9, 0.37, 0.95))
    alone = []
    for z in (x, y):
        token = torch.empty(n, dtype=torch.int32, device=DEV)
        B.mq_sample(z, t, u, token, top_p=p)
        alone.append(token)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[torch.empty(n, dtype=torch.int32, device=DEV) for _ in range(8)] for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(8):
        for k, z in enumerate((x, y)):
            with torch.cuda.stream(streams[k]):
                B.mq_sample(z, t, u, got[k][i], top_p=p)
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(g, alone[k]) for g in got[k])


@pytest.mark.parametrize("bf16", [False, True])
def test_equal_logits_beside_zero(bf16):
    """Thousands of the smallest numbers below and above zero, and of zeros of both signs, under a larger one."""
    v, tiny = 5001, 2.0 ** -133 if bf16 else 2.0 ** -149
    x = torch.full((5, v), 0.0, dtype=torch.bfloat16 if bf16 else torch.float32)
    x[0], x[1], x[2] = -tiny, tiny, -0.0
    x[3, ::2], x[3, 1::2] = -tiny, 0.0
    x[4, ::3], x[4, 1::3], x[4, 2::3] = -tiny, -0.0, tiny
    assert float(x[0, 0]) == -tiny
    x[:, 3000] = 1.0
    x, u = x.to(DEV), np.array([0.1, 0.9, 0.5, 0.99999994, 0.3], np.float32)
    for kw in (dict(k=50), dict(k=4000), dict(p=0.5), dict(k=4500, p=0.7), dict(mp=0.3), dict(mp=0.5), dict(k=4000, p=0.5, mp=0.3)):
        _check(x, 1.0, u, **kw)
    tok, _, kept = _check(x[:, :2900], 1.0, u, k=2500)
    assert kept == [2500] * 5


def _check_within_rounding(x, t, u, p):
    """top-p where single tokens weigh as little as the roundings of all weights together: with e = V 2^-44 (of the largest weight) + 2^-37 of the
    sum, running sums are off by e and borders by as much again, so the cut and the token lie where the exact sums are within 2 e of
    their borders.  The token's weight is off by 2^-44 + 2^-37 of itself, the total by e, the logarithm is rounded by 2^-24."""
    got = _run(x, t, u, p=p)
    host = x.double().cpu().numpy()
    for r, (token, logp, kept) in enumerate(zip(*got)):
        temp, want_p, draw = (float(np.float32(a[r])) for a in (t, p, u))
        w = np.exp((host[r] - host[r].max()) / temp)
        order = np.argsort(-host[r], kind="stable")
        run = np.concatenate([[0.0], np.cumsum(w[order])])
        e = w.size * 2.0 ** -44 + 2.0 ** -37 * run[-1]
        assert 1 <= kept <= w.size and run[kept - 1] < want_p * run[-1] + 2 * e and run[kept] >= want_p * run[-1] - 2 * e, (r, kept)
        cols = np.sort(order[:kept])
        run = np.concatenate([[0.0], np.cumsum(w[cols])])
        j = int(np.searchsorted(cols, token))
        assert j < cols.size and cols[j] == token, (r, token)
        assert run[j] <= draw * run[-1] + 2 * e and run[j + 1] >= draw * run[-1] - 2 * e, (r, token, run[j], draw * run[-1])
        lp = np.log(w[token] / run[-1])
        assert abs(logp - lp) <= 2.0 ** -24 * abs(lp) + 2 * (2.0 ** -44 / w[token] + 2.0 ** -37 + e / run[-1]), (r, logp, lp)
    return got


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("v,t,mid,dev", [(150001, 1.01, -20.2, 0.5), (150001, 1.0, -20.0, 0.5), (150001, 1.01, -20.3, 0.05), (150001, 1.01, -20.215, 0.001),
                                         (60013, 0.5, -10.0, 0.3), (60013, 0.503, -10.05, 0.02), (40009, 3.3, -66.0, 1.0), (1 << 20, 1.003, -20.05, 0.4)])
def test_top_p_that_ends_far_below_the_largest(bf16, v, t, mid, dev):
    """One token has nearly all of the mass, thousands lie near 20 T below it, and the nucleus ends among them: the bars of 1/32 that are counted end
    there as well, at an edge of one (T = 1, 0.5) or in its middle."""
    rng = np.random.default_rng(v + int(1000 * t))
    rows = 3 if v > 1000000 else 8
    x = (mid + dev * rng.standard_normal((rows, v))).astype(np.float32)
    x[:, 7] = 0.0
    x[1] += 70.0                        # (beyond the bars' upper end)
    x[2] += np.float32(5.0 / 64)        # (the limit elsewhere in its bar)
    x = torch.from_numpy(x).to(torch.bfloat16 if bf16 else torch.float32)
    tail = 1.0 - 1.0 / np.exp((x[0].double().numpy() - float(x[0].max())) / t).sum()      # what is not the largest one's
    share = np.array([0.5, 0.3, 0.6, 0.01, 0.9, 0.99, 0.97, 0.2])[:rows]                  # of it, within the nucleus
    p = (1.0 - tail * (1.0 - share)).astype(np.float32)
    u = np.array([0.99999994, 1 - tail / 3, 0.5, 1 - tail / 2, tail / 1000, 1 - tail / 4, 1 - tail / 5, 0.0])[:rows].astype(np.float32)
    _check_within_rounding(x.to(DEV), np.full(rows, t, np.float32), u, p)
    _check_within_rounding(x.to(DEV), np.full(rows, t, np.float32), u, np.full(rows, 0.99999994, np.float32))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("t", [0.05, 0.1, 0.3])
def test_a_nucleus_of_some_hundreds_behind_a_wrong_guess(bf16, t):
    """40 logits at one end of every interval of 1/32: they weigh less, or more, than their interval's middle, so the place of the nucleus's end is first
    guessed some intervals off, where a list of all above still fits; down to intervals that lie 20 T below the largest."""
    rng = np.random.default_rng(int(1000 * t))
    rows, v = 24, 9001
    x = np.full((rows, v), -90.0)
    for r in range(rows):
        at = rng.permutation(v)[:40 * 45].reshape(45, 40)
        for b in range(45):
            x[r, at[b]] = 2.0 - (b + 1) / 32 + (1 / 512 if r % 2 else 1 / 32 - 1 / 512)
    x = torch.from_numpy(x.astype(np.float32))
    x = (x.to(torch.bfloat16) if bf16 else x).to(DEV)
    u = rng.random(rows).astype(np.float32)
    p = np.concatenate([rng.uniform(0.3, 0.99, rows - 6), [0.995, 0.999, 0.9995, 0.9999, 0.99999, 0.999999]]).astype(np.float32)
    _check(x, t, u, p=p)
    _check(x, t, u, p=p, k=rng.integers(1300, 1700, rows))
    _check(x, t, u, p=p, mp=np.full(rows, 1e-4, np.float32))


@pytest.mark.parametrize("bf16", [False, True])
def test_min_p_beside_a_cut_among_equal_logits(bf16):
    """The first filters cut among thousands of equal logits whose weight is, within a rounding of the border, what min-p asks for: one float32 below
    the border all of them go, on it or above none."""
    v = 9001
    x = torch.full((1, v), -1.0, dtype=torch.bfloat16 if bf16 else torch.float32, device=DEV)
    x[0, 4321] = 0.0
    at = float(np.float32(np.exp(-1.0)))
    assert at > np.exp(-1.0)            # (so that the border lies above -1, by less than a float32 of logits)
    below = float(np.nextafter(np.float32(at), np.float32(0)))
    for kw in (dict(p=0.5), dict(k=5000), dict(k=5000, p=0.7), dict()):
        tok, _, kept = _check(x, 1.0, np.float32([0.7]), mp=at, **kw)
        assert (tok, kept) == ([4321], [1])
        _, _, kept = _check(x, 1.0, np.float32([0.7]), mp=below, **kw)
        assert kept[0] > 2048


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("v", [100, 2049, 30000])
def test_min_p_of_one_keeps_the_largest(bf16, v):
    """Of rows of zeros of either sign all are kept, and so are all that are as large as the largest."""
    dtype, tiny = (torch.bfloat16, 2.0 ** -133) if bf16 else (torch.float32, 2.0 ** -149)
    x = torch.zeros((5, v), dtype=dtype)
    x[1] = -0.0
    x[2, ::2] = -0.0
    x[3, 1::2] = -tiny
    x[4] = torch.finfo(dtype).min
    u = np.array([0.0, 0.99999994, 0.6, 0.3, 0.9], np.float32)
    for mp in (1.0, 5.0):
        _, _, kept = _check(x.to(DEV), 0.8, u, mp=mp)
        assert kept == [v, v, v, -(-v // 2), v]
        for kw in (dict(k=v - 1), dict(p=0.75), dict(k=v // 2, p=0.5)):
            _check(x[[0, 1, 2, 4]].to(DEV), 0.8, u[:4], mp=mp, **kw)


@pytest.mark.parametrize("top", [300.0, 1.0, 0.75, -5.5, 2.0 ** 20])
def test_masked_logits_weigh_nothing_at_any_temperature(top):
    """Temperatures at which 40 T is 1/4 to 6 steps of a float32 at the largest logit, the others masked or far below: none of their 2^17 has a share."""
    v = 1 << 17
    step = 2.0 ** (np.floor(np.log2(abs(top))) - 23)
    t = (np.linspace(0.25, 6, 47) * step / 40).astype(np.float32)
    x = torch.full((1, v), -float("inf"), device=DEV)
    x[0, 3] = top
    y = torch.full((1, v), -2.0 ** 21, device=DEV)
    y[0, 3] = top
    n = t.size
    for row, kept_all in ((x, 1), (y, v)):
        for kw in (dict(), dict(p=0.99999994), dict(k=v - 1), dict(k=v - 1, p=0.9999)):
            tok, lp, kept = _run(row.expand(n, v).contiguous(), t, np.full(n, 0.99999994, np.float32), **kw)
            assert tok == [3] * n and lp == [0.0] * n, (kw, tok, lp)
            assert kept == [1 if "p" in kw else min(kept_all, kw.get("k", v))] * n, (kw, kept)


@pytest.mark.parametrize("v", [300, 20000])
def test_infinite_temperature_beside_min_p(v):
    """Every weight is 1, which is no less than any min_p."""
    x = _logits(np.random.default_rng(v), 3, v, False)
    x[1, ::2] = -float("inf")
    for mp in (1.0, 7.0, 0.3):
        tok, _, kept = _run(x, float("inf"), np.float32([0.25, 0.5, 0.75]), mp=mp)
        assert kept == [v, v // 2, v] and tok == [v // 4, v // 2 + 1, 3 * (v // 4)]
        assert _run(x, float("inf"), np.float32([0.25, 0.5, 0.75]), mp=mp, k=100)[2] == [100] * 3
