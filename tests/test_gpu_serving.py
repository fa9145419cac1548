"""A serving run as its calls follow one another: prompts planned on the GPU, a prefix shared, steps with scaled rotary positions, attention
that reads the shared keys once, the head's logits and the next tokens drawn from them, and all of a step captured in a graph.

Attention is recomputed in float64 from the queries the GPU used and the rows that stand in the cache (tolerance: the derivation at the
attention tests, and 2^-20 for the join of two lists); tokens are the oracle's for the logits the GPU made."""
import numpy as np
import pytest
import torch

from oracle import kv_oracle as O
from oracle.sample_oracle import sample
from paper_2502_00425_b200 import binding as B
from paper_2502_00425_b200 import kvcache as KC
from paper_2502_00425_b200 import layer as LY
from paper_2502_00425_b200 import synth

from kv_util import DEV

pytestmark = pytest.mark.gpu
SHAPE = synth.LayerShape(hidden=512, n_q_heads=8, n_kv_heads=2, head_dim=128, mlp=1024)
VOCAB = 5003


def _block(seed=1, rope=True):
    blk = LY.random_block(SHAPE, seed)
    if rope:
        blk.rope = B.Rope(64, half=True, factor=4.0, original=64, fast=8.0, amp=1.1)
    return blk


def _emb(n, seed):
    return (torch.randn((n, SHAPE.hidden), generator=torch.Generator().manual_seed(seed)) * 2).to(torch.bfloat16).to(DEV)


def _cached(cache, pool, b, n):
    j = torch.arange(n)
    rows = pool.cpu()[cache.table[b].cpu().long()[j // cache.page_size], :, j % cache.page_size].double().numpy()
    if pool.dtype == torch.int8:
        rows = rows * (cache.handle.k_scale if pool is cache.K else cache.handle.v_scale).double().cpu().numpy()[:, None]
    return rows


def _check_attention(cache, tr, new, perms=None):
    q = tr.tensors["q_rope"].double().cpu().numpy().reshape(-1, SHAPE.n_q_heads, 128)
    got = tr.tensors["attn"].double().cpu().numpy().reshape(q.shape)
    at, live = 0, 0
    int8 = cache.K.dtype == torch.int8
    p_step = 2.0 ** -11 if int8 else 2.0 ** -8
    for b, (n, length) in enumerate(zip(new, cache.lengths())):
        K, V = _cached(cache, cache.K, b, length), _cached(cache, cache.V, b, length)
        perm = None if perms is None or n == 0 else perms[live].cpu().numpy()
        live += n > 0
        for h in range(SHAPE.n_q_heads):
            ref, _, _, abs_pv, mag = O.attention(q[at:at + n, h], K[:, h // 4], V[:, h // 4], 128 ** -0.5, perm)
            ds = (128 + 8) * 2.0 ** -23 * mag[:, None]
            tol = 2.0 ** -8 * np.abs(ref) + (p_step + 2 * ds + 2.0 ** -19 + 2.0 ** -20) * abs_pv + 1e-30
            if int8:
                tol = tol + 2.0 ** -31 * np.abs(V[:, h // 4]).sum(0)
            assert np.all(np.abs(got[at:at + n, h] - ref) <= tol)
        at += n


def _calibrated(blk):
    blk.forward_cached([_emb(40, 9)], KC.PagedKVCache(1, 10, 100, 2, 128, 16), calibrate=True)
    return blk


@pytest.mark.parametrize("int8", [False, True])
def test_shared_prompt_and_answers(int8):
    blk = _calibrated(_block())
    scales = (torch.full((2,), 0.02, device=DEV), torch.full((2,), 0.05, device=DEV)) if int8 else (None, None)
    cache = KC.DeviceKVCache(5, 60, 300, 2, 128, 16, *scales, shared_from=0)
    prompt = _emb(90, 1)
    none = _emb(0, 1)
    _, tr = blk.forward_cached([prompt, none, none, none, _emb(7, 2)], cache)      # one prompt, and a stranger
    _check_attention(cache, tr, [90, 0, 0, 0, 7])
    assert cache.share(0, 1, 3) == 80
    tails = [_emb(n, 30 + n) for n in (3, 12, 5, 1)]
    for b in range(3):
        tails[b] = torch.cat([prompt[80:], tails[b]])
    new = [0] + [t.shape[0] for t in tails]
    _, tr = blk.forward_cached([none] + tails, cache)                            # the rest of the prompt and their questions
    _check_attention(cache, tr, new)
    assert cache.lengths() == [90, 93, 102, 95, 8]
    for step in range(3):                                                        # answers, the prompt's own sequence going on as well
        _, tr = blk.forward_cached([_emb(1, 60 + 5 * step + b) for b in range(5)], cache)
        _check_attention(cache, tr, [1] * 5)
    # the keys of the shared pages are those a cache without sharing holds
    alone = KC.PagedKVCache(1, 10, 150, 2, 128, 16, *scales)
    blk.forward_cached([torch.cat([prompt, _emb(12, 42)])], alone)
    rows = _cached(cache, cache.K, 2, 102)
    j = torch.arange(102)
    want = alone.K.cpu()[torch.tensor(alone.pages[0])[j // 16], :, j % 16].double().numpy()
    assert np.array_equal(rows, want * 0.02 if int8 else want) or np.allclose(rows, want * (np.float64(np.float32(0.02)) if int8 else 1.0), rtol=1e-12)
    cache.release([1, 2, 3])
    _, tr = blk.forward_cached([_emb(2, 80), _emb(33, 81), none, none, _emb(1, 82)], cache)   # and a new sequence in a freed place
    _check_attention(cache, tr, [2, 33, 0, 0, 1])
    assert cache.lengths() == [95, 33, 0, 0, 12] and cache.status_ok() and blk.device_status_ok()


def test_image_turns_behind_a_shared_prompt():
    blk = _calibrated(_block(3, rope=False))
    cache = KC.DeviceKVCache(3, 40, 300, 2, 128, 32, shared_from=0)
    vis = lambda *runs: torch.cat([torch.full((n,), v, dtype=torch.uint8) for v, n in runs]).to(DEV)
    _, tr = blk.forward_cached([_emb(70, 1), _emb(0, 1), _emb(0, 1)], cache, [vis((0, 10), (1, 50), (0, 10)), None, None])
    _check_attention(cache, tr, [70, 0, 0], tr.perms)
    assert cache.share(0, 1, 2) == 64
    chunks = [_emb(3, 2), _emb(40, 3), _emb(21, 4)]
    _, tr = blk.forward_cached(chunks, cache, [None, vis((0, 4), (1, 30), (0, 6)), vis((1, 20), (0, 1))])
    _check_attention(cache, tr, [3, 40, 21], tr.perms)
    assert cache.status_ok()


def _draws(rng, n):
    f = lambda a, b: torch.from_numpy(rng.uniform(a, b, n).astype(np.float32)).to(DEV)
    return dict(temperature=f(0.5, 1.5), u=f(0, 1), top_k=torch.from_numpy(rng.integers(1, 300, n).astype(np.int32)).to(DEV), top_p=f(0.5, 0.99),
                min_p=f(0, 0.05))


def test_head_logits_and_tokens():
    head, rng = LY.random_head(SHAPE.hidden, VOCAB, 4), np.random.default_rng(4)
    assert head.w.N == 5008
    for n in (1, 2, 9):
        x, par = _emb(n, 70 + n), _draws(rng, n)
        logp, kept = torch.empty(n, device=DEV), torch.empty(n, dtype=torch.int32, device=DEV)
        token = head.next_tokens(x, logp=logp, kept=kept, **par)
        logits = head.logits(x)
        assert logits.shape == (n, VOCAB) and logits.dtype == torch.float32
        h = torch.empty_like(x)
        B.mq_glue_rmsnorm(x, head.gain, h)
        y = torch.empty((n, head.w.N), device=DEV)
        B.mq_w4a8_msq_linear(h, head._seg, head.w.s_vis, head.w.s_txt, head.w.layout, head.w.s_w, y, B.new_workspace(n, 512, 5008), 5008)
        assert torch.equal(y[:, :VOCAB], logits)
        host = {k: v.cpu().numpy() for k, v in par.items()}
        for r in range(n):
            want, lp, keep = sample(logits[r].cpu().numpy(), host["temperature"][r], host["u"][r], host["top_k"][r], host["top_p"][r], host["min_p"][r])
            assert (int(token[r]), int(kept[r])) == (want, keep.size) and abs(float(logp[r]) - lp) <= 2.0 ** -24 * abs(lp) + 2.0 ** -30
    assert head.logits(_emb(0, 1)).shape == (0, VOCAB) and head.device_status_ok()
    with pytest.raises(ValueError):
        LY.W4A8Head(head.w, head.gain, 5009)


def test_a_captured_step_goes_on_by_itself():
    """Embedding lookup, plan, block, head and draw in one graph, replayed: the tokens and the cache are those of steps made one by one."""
    blk, head = _calibrated(_block(5)), LY.random_head(SHAPE.hidden, VOCAB, 6)
    table = _emb(VOCAB, 11)
    n, steps = 4, 6
    rng = np.random.default_rng(8)
    par = _draws(rng, n)
    us = [torch.from_numpy(rng.random(n).astype(np.float32)).to(DEV) for _ in range(steps + 1)]
    out = []
    for captured in (False, True):
        cache = KC.DeviceKVCache(n, 60, 200, 2, 128, 16, shared_from=0)
        blk.forward_cached([_emb(60, 1), _emb(0, 1), _emb(0, 1), _emb(19, 2)], cache)
        cache.share(0, 1, 2)
        blk.forward_cached([_emb(0, 1), _emb(4, 3), _emb(9, 4), _emb(0, 1)], cache)
        tokens = torch.tensor([1, 2, 3, 4], dtype=torch.int32, device=DEV)

        def step():
            rows, _ = blk.forward_cached(list(table[tokens.long()].split(1)), cache)
            tokens.copy_(head.next_tokens(torch.cat(rows), **par))

        par["u"].copy_(us[0])
        step()                                  # (makes workspaces and sizes)
        history = [tokens.tolist()]
        graph = None
        if captured:
            keep = (tokens.clone(), cache.kv_len.clone())
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
            assert torch.equal(tokens, keep[0]) and torch.equal(cache.kv_len, keep[1])   # (recorded, not run)
        for k in range(steps):
            par["u"].copy_(us[k + 1])
            graph.replay() if captured else step()
            torch.cuda.synchronize()
            history.append(tokens.tolist())
        out.append((history, cache.lengths(), cache.K.clone(), cache.V.clone(), cache.table.clone()))
        assert cache.status_ok() and blk.device_status_ok() and head.device_status_ok()
    a, b = out
    assert a[0] == b[0] and a[1] == b[1] == [61 + steps, 53 + steps, 58 + steps, 20 + steps]
    assert torch.equal(a[2], b[2]) and torch.equal(a[3], b[3]) and torch.equal(a[4], b[4])


def test_a_step_that_cannot_be_made_shows_in_the_status():
    blk = _calibrated(_block(2))
    cache = KC.DeviceKVCache(2, 4, 100, 2, 128, 16)
    blk.forward_cached([_emb(20, 1), _emb(20, 2)], cache)
    before = (cache.K.clone(), cache.lengths())
    assert cache.status_ok()
    blk.forward_cached([_emb(20, 3), _emb(1, 4)], cache)          # five pages are needed, four there are
    assert not cache.status_ok() and cache.plan_status.tolist() == [B.MQ_ERR_WORKSPACE, 4]
    assert cache.lengths() == before[1] and torch.equal(cache.K, before[0])
    cache.plan_status.zero_()
    _, tr = blk.forward_cached([_emb(1, 3), _emb(1, 4)], cache)
    _check_attention(cache, tr, [1, 1])
    assert cache.status_ok()


def test_a_failing_step_is_taken_back(monkeypatch):
    blk = _calibrated(_block(6))
    cache = KC.DeviceKVCache(2, 20, 100, 2, 128, 16)
    blk.forward_cached([_emb(20, 1), _emb(5, 2)], cache)
    before = (cache.lengths(), cache.free[:int(cache.n_free)].tolist(), cache.seen.tolist())
    with monkeypatch.context() as m:
        m.setattr(LY.B, "mq_kv_attention", lambda *a, **k: (_ for _ in ()).throw(RuntimeError("out of memory")))
        with pytest.raises(RuntimeError, match="out of memory"):
            blk.forward_cached([_emb(30, 3), _emb(1, 4)], cache)
    assert before == (cache.lengths(), cache.free[:int(cache.n_free)].tolist(), cache.seen.tolist()) and cache.status_ok()


def test_a_step_of_new_sizes_is_not_captured():
    cache = KC.DeviceKVCache(2, 20, 100, 2, 128, 16)
    g = torch.cuda.CUDAGraph()
    with pytest.raises(RuntimeError, match="once before"):
        with torch.cuda.graph(g):
            cache.extend([1, 1])


@pytest.mark.parametrize("int8", [False, True])
def test_answers_that_end_one_after_another(int8, monkeypatch):
    """Questions about one prompt, of which some end and leave their places empty or to new sequences: the others go on reading the shared keys once."""
    blk = _calibrated(_block(7))
    scales = (torch.full((2,), 0.02, device=DEV), torch.full((2,), 0.05, device=DEV)) if int8 else (None, None)
    cache = KC.DeviceKVCache(7, 80, 300, 2, 128, 16, *scales, shared_from=0)
    groups = []
    call = B.mq_kv_attention_shared
    monkeypatch.setattr(B, "mq_kv_attention_shared", lambda *a, **k: (groups.append(a[4].tolist()), call(*a, **k))[1])
    none = _emb(0, 1)
    blk.forward_cached([_emb(90, 1)] + [none] * 6, cache)
    assert cache.share(0, 1, 6) == 80

    def step(rows, seed):
        _, tr = blk.forward_cached([_emb(n, seed + b) for b, n in enumerate(rows)], cache)
        _check_attention(cache, tr, rows)
        return groups[-1]

    assert step([0, 5, 3, 9, 1, 2, 4], 10) == [0] * 7
    cache.release([2])
    assert step([1, 1, 0, 1, 1, 1, 1], 20) == [0] * 7
    cache.release([4, 5])
    assert step([1, 1, 0, 1, 0, 0, 1], 30) == [0] * 7
    assert step([0, 1, 20, 1, 0, 0, 1], 40) == [0, 0, 2, 3, 3, 3, 3]          # a new sequence in place 2
    assert step([1, 1, 1, 1, 7, 0, 1], 50) == [0, 0, 2, 3, 4, 5, 6]           # and in place 4
    cache.release([2, 4])
    assert step([1, 1, 0, 1, 0, 0, 1], 60) == [0] * 7
    assert cache.status_ok() and blk.device_status_ok()


def test_a_step_of_new_lengths_waits_for_nothing():
    """Lengths that were never asked for go to the GPU behind what is queued, and the host goes on."""
    cache = KC.DeviceKVCache(16, 200, 400, 2, 128, 16)
    lengths, rng = [0] * 16, np.random.default_rng(12)
    for _ in range(3):                                  # (the first rounds make the pinned memory)
        torch.cuda.synchronize()
        done = torch.cuda.Event()
        torch.cuda._sleep(200_000_000)                  # some 0.1 s
        done.record()
        for _ in range(4):
            new, keep = rng.integers(0, 3, 16).tolist(), rng.integers(0, 9, 16).tolist()
            cache.extend(new, keep)
            lengths = [min(k, l) + a for k, l, a in zip(keep, lengths, new)]
        ahead = not done.query()
    assert ahead and cache.lengths() == lengths and cache.status_ok()


def test_lengths_stay_until_another_stream_has_read_them():
    """Lengths made on one stream and read on another one, which is behind: they are dropped from the cache, and their memory is asked for, in between."""
    cache = KC.DeviceKVCache(16, 200, 400, 2, 128, 16)
    cache.extend([3] * 16)
    cache.extend([0] * 16, keep=[0] * 16)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
        cache.extend([3] * 16)                                  # (the arrays that the default stream made)
        for i in range(300):
            cache.extend([0] * 16, keep=[1 << 30] * 15 + [1000 + i])
    assert (3,) * 16 not in cache._numbers
    taken = [torch.full((16,), 2, dtype=torch.int32, device=DEV) for _ in range(400)]
    torch.cuda.synchronize()
    assert cache.lengths() == [3] * 16 and cache.status_ok() and len(taken) == 400
