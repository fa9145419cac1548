"""A decoder block that goes on after its prompt: projections, norm + rotary + store, attention over the paged cache,
accumulated weights and eviction as they follow one another.  Every attention is recomputed in float64 from the queries
the GPU used and the rows that stand in the cache (tolerance: the derivation at the attention tests)."""
import numpy as np
import pytest
import torch

from oracle import kv_oracle as O
from paper_2502_00425_b200 import binding as B
from paper_2502_00425_b200 import kvcache as KC
from paper_2502_00425_b200 import layer as LY
from paper_2502_00425_b200 import synth

from kv_util import DEV

pytestmark = pytest.mark.gpu
SHAPE = synth.LayerShape(hidden=512, n_q_heads=8, n_kv_heads=2, head_dim=128, mlp=1024)


def _block(seed=1, norms=False):
    blk = LY.random_block(SHAPE, seed)
    if norms:
        g = torch.Generator().manual_seed(seed)
        blk.g_q, blk.g_k = (1 + 0.2 * torch.randn(128, generator=g)).to(DEV), (1 + 0.2 * torch.randn(128, generator=g)).to(DEV)
    return blk


def _emb(n, seed):
    return (torch.randn((n, SHAPE.hidden), generator=torch.Generator().manual_seed(seed)) * 2).to(torch.bfloat16).to(DEV)


def _cached(cache, pool, b):
    """The rows of sequence b in the cache, as numbers: float64 [keys, heads, dim]."""
    j = torch.arange(cache.lengths[b])
    pages = torch.tensor(cache.pages[b], dtype=torch.long)[j // cache.page_size]
    rows = pool.cpu()[pages, :, j % cache.page_size].double().numpy()
    if pool.dtype == torch.int8:
        rows = rows * (cache.handle.k_scale if pool is cache.K else cache.handle.v_scale).double().cpu().numpy()[:, None]
    return rows


def _check_attention(cache, tr, new, perms=None):
    """tr.tensors["attn"] against the float64 attention over what the cache holds; returns the softmax weights per (b, g) and
    by how much of themselves the float32 ones may be off: twice the score's error (the log-sum-exp has it too), the roundings
    of score and log-sum-exp in the exponent's argument, exp2, and the sum."""
    q = tr.tensors["q_rope"].double().cpu().numpy().reshape(-1, SHAPE.n_q_heads, 128)
    got = tr.tensors["attn"].double().cpu().numpy().reshape(q.shape)
    group, at, w, rel = SHAPE.n_q_heads // SHAPE.n_kv_heads, 0, {}, 0.0
    p_step = 2.0 ** -11 if cache.K.dtype == torch.int8 else 2.0 ** -8
    k_live = 0
    for b, n in enumerate(new):
        K, V = _cached(cache, cache.K, b), _cached(cache, cache.V, b)
        perm = None if perms is None or n == 0 else perms[k_live].cpu().numpy()
        k_live += n > 0
        for h in range(SHAPE.n_q_heads):
            ref, _, p, abs_pv, mag = O.attention(q[at:at + n, h], K[:, h // group], V[:, h // group], 128 ** -0.5, perm)
            ds = (128 + 8) * 2.0 ** -23 * mag[:, None]
            tol = 2.0 ** -8 * np.abs(ref) + (p_step + 2 * ds + 2.0 ** -19) * abs_pv + 1e-30
            if p_step < 2.0 ** -8:
                tol = tol + 2.0 ** -31 * np.abs(V[:, h // group]).sum(0)
            assert np.all(np.abs(got[at:at + n, h] - ref) <= tol)
            w[b, h // group] = w.get((b, h // group), 0) + p.sum(0)
            if n:
                rel = max(rel, 2 * ds.max() + 2.0 ** -21 * (mag.max() + np.log(len(K)) + 1) + n * group * 2.0 ** -24)
        at += n
    return w, rel


def test_prompt_in_turns_equals_prompt_at_once_and_decode_goes_on():
    blk = _block(norms=True)
    lens = [90, 33, 1]
    embs = [_emb(n, 10 + b) for b, n in enumerate(lens)]
    blk.forward_cached(embs, KC.PagedKVCache(3, 24, 200, 2, 128, page_size=16), calibrate=True)   # sets the static scales
    two = KC.PagedKVCache(3, 24, 200, 2, 128, page_size=16)
    half = [[e[:40] if b == 0 else e[:0] if b == 1 else e for b, e in enumerate(embs)],
            [e[40:] if b == 0 else e if b == 1 else e[:0] for b, e in enumerate(embs)]]
    one = KC.PagedKVCache(3, 24, 200, 2, 128, page_size=16)
    outs, tr = blk.forward_cached(embs, one)
    _check_attention(one, tr, lens)
    for part in half:
        _, tr = blk.forward_cached(part, two)
        _check_attention(two, tr, [e.shape[0] for e in part])
    assert one.lengths == two.lengths == lens
    for b in range(3):
        # the linears and the norm are exact per row, so the cache holds the same rows however the prompt came
        for x, y in ((one.K, two.K), (one.V, two.V)):
            assert np.array_equal(_cached(one, x, b), _cached(two, y, b))
    for step in range(3):
        toks = [_emb(1, 50 + 3 * step + b) for b in range(3)]
        o1, tr1 = blk.forward_cached(toks, one)
        o2, tr2 = blk.forward_cached(toks, two)
        _check_attention(one, tr1, [1, 1, 1])
        for a, c in zip(o1, o2):
            assert torch.equal(a, c)      # the page numbers differ, the rows do not
    assert one.status_ok() and two.status_ok() and blk.device_status_ok()
    empty, _ = blk.forward_cached([e[:0] for e in embs], one)
    assert [e.shape[0] for e in empty] == [0, 0, 0]


def test_image_turns_in_aifs_order():
    """Each turn is reordered on its own (visual tokens first); the result equals the causal turn in the original order."""
    blk = _block(2)
    is_vis = [torch.tensor([0] * 7 + [1] * 50 + [0] * 13, dtype=torch.uint8, device=DEV), torch.tensor([1] * 20 + [0] * 4, dtype=torch.uint8, device=DEV)]
    embs = [_emb(70, 3), _emb(24, 4)]
    cache = KC.PagedKVCache(2, 20, 200, 2, 128, page_size=32)
    blk.forward_cached(embs, KC.PagedKVCache(2, 20, 200, 2, 128, page_size=32), is_vis, calibrate=True)
    outs, tr = blk.forward_cached(embs, cache, is_vis)
    _check_attention(cache, tr, [70, 24], tr.perms)
    # the whole block without a cache, on the same scales: same linears, attention by mq_aifs_attention
    ref, tr0 = blk.forward_batch(embs, is_vis)
    assert torch.equal(tr0.tensors["emb_u"], tr.tensors["emb_u"])
    a, c = tr0.tensors["attn"].float(), tr.tensors["attn"].float()
    assert float(((a - c).abs().amax(1) / a.abs().amax(1)).max()) < 4e-2       # two kernels, each within 2e-2 of the exact row
    # the next turn, its image behind the first one's text
    outs, tr = blk.forward_cached([_emb(40, 5), _emb(9, 6)], cache, [torch.tensor([0] * 5 + [1] * 30 + [0] * 5, dtype=torch.uint8, device=DEV),
                                                                     torch.zeros(9, dtype=torch.uint8, device=DEV)])
    assert cache.lengths == [110, 33] and [o.shape[0] for o in outs] == [40, 9]
    _check_attention(cache, tr, [40, 9], tr.perms)
    assert cache.status_ok()


@pytest.mark.parametrize("int8", [False, True])
def test_weights_eviction_and_going_on(int8):
    blk = _block(7)
    scales = (torch.full((2,), 0.02, device=DEV), torch.full((2,), 0.05, device=DEV)) if int8 else (None, None)
    cache = KC.PagedKVCache(2, 40, 300, 2, 128, 16, *scales)
    blk.forward_cached([_emb(5, 1), _emb(5, 2)], KC.PagedKVCache(2, 40, 300, 2, 128, 16), calibrate=True)
    cache.track_weights()
    lens, total = [150, 30], {}
    _, tr = blk.forward_cached([_emb(n, 20 + n) for n in lens], cache)
    total, rel = _check_attention(cache, tr, lens)
    for step in range(4):
        _, tr = blk.forward_cached([_emb(1, 60 + step), _emb(1, 70 + step)], cache)
        more, r = _check_attention(cache, tr, [1, 1])
        rel = max(rel, r) + 2.0 ** -23
        for key, w in more.items():
            total[key] = np.concatenate([total[key], np.zeros(len(w) - len(total[key]))]) + w
    for (b, g), w in total.items():
        got = cache.weights[b, g, :len(w)].double().cpu().numpy()
        assert np.all(np.abs(got - w) <= rel * w + 1e-30)
    before = [(_cached(cache, cache.K, b), _cached(cache, cache.V, b)) for b in range(2)]
    had = cache.weights.clone().cpu().numpy()
    n_before, free = list(cache.lengths), len(cache.free)
    kept = cache.evict(64, 4, 16).cpu().numpy()
    assert cache.lengths == [64, 34] and cache.tokens == [154, 34]
    assert len(cache.free) > free
    for b in range(2):
        K, V = _cached(cache, cache.K, b), _cached(cache, cache.V, b)
        for g in range(2):
            ref = O.keep(had[b, g, :n_before[b]], n_before[b], 64, 4, 16)
            assert np.array_equal(kept[b, g, :len(ref)], ref)
            assert np.array_equal(K[:, g], before[b][0][ref, g]) and np.array_equal(V[:, g], before[b][1][ref, g])
            assert np.array_equal(cache.weights[b, g, :len(ref)].cpu().numpy(), had[b, g, ref])
            assert not cache.weights[b, g, len(ref):].any()
    _, tr = blk.forward_cached([_emb(1, 90), _emb(3, 91)], cache)
    _check_attention(cache, tr, [1, 3])
    assert cache.tokens == [155, 37] and cache.status_ok()


def test_cache_refusals():
    cache = KC.PagedKVCache(2, 3, 64, 2, 128, page_size=16)
    with pytest.raises(RuntimeError):
        cache.extend([70, 0])                # longer than the cache was made for
    with pytest.raises(RuntimeError):
        cache.extend([40, 10])               # four pages are needed, three are there
    assert cache.lengths == [0, 0] and len(cache.free) == 3
    with pytest.raises(RuntimeError):
        cache.evict(8, 0, 0)                 # no weights are tracked


@pytest.mark.parametrize("n_new", [1, 40])
def test_a_failed_accumulation_of_weights_shows_in_the_status(n_new):
    cache = KC.PagedKVCache(2, 30, 130, 2, 128, page_size=16)
    cache.track_weights()
    q = _emb(2 * n_new, 3)[:, :512].repeat(1, 2).contiguous()
    cache.attend(q, cache.extend([n_new, n_new]), 8)
    assert cache.status_ok()
    cache.weights = torch.zeros((2, 2, 2 * n_new - 1), device=DEV)     # rows too short for what follows: the call leaves keys out and says so
    cache.attend(q, cache.extend([n_new, n_new]), 8)
    assert not cache.status_ok()
    assert all(B.mq_last_device_status(ws)[0] == B.MQ_OK for ws in cache._ws.values())
    with pytest.raises(RuntimeError, match="not whole"):
        cache.evict(2, 0, 1)
    cache.track_weights()                                          # starts over
    assert cache.status_ok()
    cache.attend(q, cache.extend([n_new, n_new]), 8)
    cache.evict(2, 0, 1)
    assert cache.lengths == [2, 2] and cache.status_ok()


def test_workspaces_of_a_cache_stay_few_and_are_made_before_a_capture():
    cache = KC.PagedKVCache(2, 64, 2000, 2, 128, 64, device=DEV)
    q = lambda n: _emb(n, 3)[:, :512].repeat(1, 2).contiguous()
    for n in list(range(1, 60, 3)) + [200, 300, 500]:
        step = cache.extend([n, 1])
        cache.attend(q(n + 1), step, 8)
    assert len(cache._ws) <= 6 and cache.status_ok()
    new = KC.PagedKVCache(1, 4, 200, 2, 128, 64, device=DEV)
    step, rows = new.extend([1]), q(1)
    g = torch.cuda.CUDAGraph()
    with pytest.raises(RuntimeError, match="once before"):
        with torch.cuda.graph(g):
            new.attend(rows, step, 8)
    new.attend(rows, step, 8)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        o = new.attend(rows, step, 8)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(o, new.attend(rows, step, 8)) and new.status_ok()


@pytest.mark.parametrize("images", [False, True])
def test_a_step_that_fails_leaves_the_cache_as_it_was(images, monkeypatch):
    """An error behind the attention, and one in it: the same call made again gives what it gives without the failures."""
    blk = _block(9)
    vis = (lambda *ns: [torch.tensor([0] + [1] * (n - 1), dtype=torch.uint8, device=DEV) for n in ns]) if images else (lambda *ns: None)
    steps = [([_emb(70, 1), _emb(24, 2)], vis(70, 24)), ([_emb(20, 3), _emb(9, 4)], vis(20, 9)), ([_emb(1, 5), _emb(1, 6)], vis(1, 1))]
    blk.forward_cached(*steps[0][:1], KC.PagedKVCache(2, 30, 200, 2, 128, 16), steps[0][1], calibrate=True)
    got = []
    for fail in (False, True):
        cache = KC.PagedKVCache(2, 30, 200, 2, 128, 16)
        cache.track_weights()
        outs = []
        for embs, v in steps:
            if fail:
                before = (list(cache.free), [list(p) for p in cache.pages], list(cache.lengths), list(cache.tokens), cache.weights.clone())
                for where, name in ((blk, "_behind_attention"), (LY.B, "mq_kv_attention"), (LY.B, "mq_qk_norm_rope"), (LY.B, "mq_kv_weights")):
                    with monkeypatch.context() as m:
                        def fails(*a, **k):
                            raise RuntimeError("out of memory")
                        m.setattr(where, name, fails)
                        with pytest.raises(RuntimeError, match="out of memory"):
                            blk.forward_cached(embs, cache, v)
                    assert before[:4] == (cache.free, cache.pages, cache.lengths, cache.tokens) and torch.equal(cache.weights, before[4])
            outs += blk.forward_cached(embs, cache, v)[0]
        got.append((outs, cache))
    (a, ca), (b, cb) = got
    assert all(torch.equal(x, y) for x, y in zip(a, b)) and ca.pages == cb.pages and ca.lengths == cb.lengths
    assert torch.equal(ca.weights, cb.weights) and bool((ca.weights > 0).any()) and ca.status_ok() and cb.status_ok()


def test_turns_of_text_beside_turns_with_images():
    """None in place of a chunk's modalities: text only, as zeros say."""
    blk = _block(5)
    embs = [_emb(40, 1), _emb(24, 2), _emb(1, 3)]
    vis = torch.tensor([0] * 3 + [1] * 30 + [0] * 7, dtype=torch.uint8, device=DEV)
    blk.forward_cached(embs, KC.PagedKVCache(3, 20, 100, 2, 128, 16), [vis] + [torch.zeros(e.shape[0], dtype=torch.uint8, device=DEV) for e in embs[1:]],
                       calibrate=True)
    got = []
    for text in (None, torch.zeros):
        is_vis = [vis] + [None if text is None else text(e.shape[0], dtype=torch.uint8, device=DEV) for e in embs[1:]]
        cache = KC.PagedKVCache(3, 20, 100, 2, 128, 16)
        got.append((blk.forward_cached(embs, cache, is_vis)[0], cache.K.clone(), cache.V.clone()))
        assert cache.status_ok()
    assert all(torch.equal(a, b) for a, b in zip(got[0][0], got[1][0])) and torch.equal(got[0][1], got[1][1]) and torch.equal(got[0][2], got[1][2])
