"""The key/value-cache operators as a serving program uses them, for measurement.

Four operators around one paged cache:

  append   RMSNorm of every query and key head (optional gains), the rotary embedding, and the store of K and V into
           the cache's pages, in one pass over the projections' outputs;
  attend   grouped-query attention of each sequence's new tokens (one, a few, or a long chunk) over its paged cache,
           in token order or in AIFS order (visual tokens of the chunk first);
  weights  the softmax weight every cached key has received, accumulated over calls, per key/value head;
  evict    the cache cut down to a budget of keys per key/value head by that weight, copied to fresh pages in order.

`own` false: the plain form, elementary torch operations in 32 bits (64 for the rotary angles).  `own` true: the
library's entry points.  `exact` is the definition in 64 bits, one sequence and key/value head at a time.
"""
import math

import torch

own = False
DEV = "cuda"


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one decode step of 32 sequences: 32 rows, where the launch is most of the time
        dict(name="append decode 32", op="append", batch=32, new=1, ctx=500, hq=28, hkv=4, dim=128, page=64,
             norm=True, half=False),
        # the prompts of the 4 x 2432-token batch (visual tiles and text), 32 / 8 heads
        dict(name="append prompt 9728", op="append", batch=4, new=2432, ctx=0, hq=32, hkv=8, dim=128, page=128,
             norm=True, half=True),
        # one sequence decoding behind the 3360-token prompt of three images: latency
        dict(name="decode 1 x 3361", op="attend", batch=1, new_lo=1, new_hi=1, ctx_lo=3360, ctx_hi=3360, hq=28, hkv=4,
             dim=128, page=64, int8=False, aifs=False),
        # a serving batch of very different lengths, one new token each
        dict(name="decode 64 ragged", op="attend", batch=64, new_lo=1, new_hi=1, ctx_lo=63, ctx_hi=8191, hq=32, hkv=8,
             dim=128, page=16, int8=False, aifs=False),
        # the same batch on an 8-bit cache
        dict(name="decode 64 ragged int8", op="attend", batch=64, new_lo=1, new_hi=1, ctx_lo=63, ctx_hi=8191, hq=32,
             hkv=8, dim=128, page=64, int8=True, aifs=False),
        # follow-up turns, each with an image in it: the new rows stand in AIFS order behind the cached context
        dict(name="turns aifs", op="attend", batch=6, new_lo=40, new_hi=701, ctx_lo=200, ctx_hi=4001, hq=32, hkv=8,
             dim=128, page=64, int8=False, aifs=True),
        # a middle-sized chunk over an 8-bit cache of 64-wide heads
        dict(name="chunk int8 dim 64", op="attend", batch=3, new_lo=100, new_hi=257, ctx_lo=1000, ctx_hi=6001, hq=16,
             hkv=2, dim=64, page=32, int8=True, aifs=False),
        # one chunk of a long prompt behind 32768 cached tokens: the largest
        dict(name="chunk 2048 over 32768", op="attend", batch=1, new_lo=2048, new_hi=2048, ctx_lo=32768, ctx_hi=32768,
             hq=28, hkv=4, dim=128, page=128, int8=False, aifs=False),
        # the accumulated weights after a decode step
        dict(name="weights decode 32", op="weights", batch=32, new_lo=1, new_hi=1, ctx_lo=255, ctx_hi=4095, hq=28, hkv=4,
             dim=128, page=64, int8=False, aifs=False),
        # the accumulated weights of a chunk
        dict(name="weights chunk 1024", op="weights", batch=2, new_lo=900, new_hi=1024, ctx_lo=2000, ctx_hi=8192, hq=32,
             hkv=8, dim=128, page=64, int8=False, aifs=False),
        # four sequences behind an image prompt cut to 1024 keys
        dict(name="evict 4 to 1024", op="evict", batch=4, len_lo=2500, len_hi=3361, hq=28, hkv=4, dim=128, page=64,
             budget=1024, first=4, last=128, int8=False),
        # a whole batch cut at once, some sequences already within the budget
        dict(name="evict 32 to 2000", op="evict", batch=32, len_lo=700, len_hi=16384, hq=32, hkv=8, dim=128, page=64,
             budget=2000, first=16, last=500, int8=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    hq, hkv = rng.choice([(28, 4), (32, 8)])
    dim = rng.choice([128, 128, 64])
    page = rng.choice([16, 32, 64, 128])
    op = rng.choice(["append", "attend", "attend", "attend", "weights", "evict"])
    case = dict(op=op, hq=hq, hkv=hkv, dim=dim, page=page)
    if op == "append":
        batch = _log_int(rng, 1, 64)
        new = _log_int(rng, 1, max(1, 9728 // batch))
        case.update(batch=batch, new=new, ctx=rng.randrange(0, 300), norm=rng.random() < 0.7, half=rng.random() < 0.5)
    elif op == "evict":
        lo, hi = sorted((_log_int(rng, 200, 16384), _log_int(rng, 200, 16384)))
        budget = _log_int(rng, 100, 4096)
        first = rng.randrange(0, 1 + min(16, budget // 8))
        case.update(batch=_log_int(rng, 1, 32), len_lo=lo, len_hi=hi, budget=budget, first=first,
                    last=rng.randrange(0, 1 + budget // 3), int8=rng.random() < 0.3)
    else:
        if rng.random() < 0.5:   # decode: one or a few new tokens each
            batch = _log_int(rng, 1, 64)
            new_lo, new_hi = 1, rng.choice([1, 1, 3])
            lo, hi = sorted((_log_int(rng, 1, 8191), _log_int(rng, 16, 8191)))
        else:                    # chunks
            batch = _log_int(rng, 1, 6)
            new_lo, new_hi = sorted((_log_int(rng, 1, 1024), _log_int(rng, 16, 1024)))
            lo, hi = sorted((_log_int(rng, 1, 8192), _log_int(rng, 16, 8192)))
        case.update(batch=batch, new_lo=new_lo, new_hi=new_hi, ctx_lo=lo, ctx_hi=hi, int8=rng.random() < 0.35,
                    aifs=new_hi > 3 and rng.random() < 0.35)
    return case


def _spread(lo, hi, n, phase):
    """n lengths from lo to hi, evenly over their logarithm, in a mixed-up order; both ends are among them when n > 1."""
    if n == 1:
        return [hi]
    vals = [int(round(math.exp(math.log(lo) + (math.log(hi) - math.log(lo)) * i / (n - 1)))) for i in range(n)]
    step = next(s for s in range(n // 2 + 1 + phase, 4 * n) if math.gcd(s, n) == 1)
    return [vals[(i * step + phase) % n] for i in range(n)]


def _lens(case):
    """(new tokens, total keys) of every sequence."""
    n = case["batch"]
    if case["op"] == "append":
        return [case["new"]] * n, [case["ctx"] + case["new"]] * n
    if case["op"] == "evict":
        return [0] * n, _spread(case["len_lo"], case["len_hi"], n, 1)
    new = _spread(case["new_lo"], case["new_hi"], n, 0)
    ctx = _spread(case["ctx_lo"], case["ctx_hi"], n, 1)
    return new, [a + b for a, b in zip(new, ctx)]


def work(case):
    new, tot = _lens(case)
    hq, hkv, d = case["hq"], case["hkv"], case["dim"]
    t = sum(new)
    if case["op"] == "append":
        # q, k, v read; q, k, v written (bf16); positions, slots
        return {"bytes": t * (2 * (hq + 2 * hkv) * d * 2 + 12), "flops": t * (hq + hkv) * d * 10}
    es = 1 if case["int8"] else 2
    if case["op"] == "evict":
        kept = sum(min(n, case["budget"]) for n in tot) * hkv
        # every weight read; kept K and V rows read and written; their indices written
        return {"bytes": sum(tot) * hkv * 4 + kept * (4 * d * es + 4 + 4), "flops": sum(tot) * hkv}
    pairs = sum(n * (k - n) + n * (n + 1) // 2 for n, k in zip(new, tot))
    if case["op"] == "weights":
        # queries, their log-sum-exp, K once, the weights read and written
        return {"bytes": t * hq * (2 * d + 4) + sum(tot) * hkv * (d * es + 8), "flops": 2 * d * hq * pairs}
    return {"bytes": t * hq * (4 * d + 4) + sum(tot) * hkv * 2 * d * es, "flops": 4 * d * hq * pairs}


# ------------------------------------------------------------------------------------------------ inputs
def _chunk_order(n):
    """AIFS order of a chunk [text][image][text]: its visual tokens first, then its text tokens."""
    a, b = n // 5, n - n // 4
    return list(range(a, b)) + list(range(a)) + list(range(b, n))


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    new, tot = _lens(case)
    hq, hkv, d, page, batch = case["hq"], case["hkv"], case["dim"], case["page"], case["batch"]
    n_pages = [-(-n // page) for n in tot]
    width = max(n_pages) + 1
    order = torch.randperm(sum(n_pages), generator=g, device=DEV, dtype=torch.int32)
    table = torch.full((batch, width), -1, dtype=torch.int32, device=DEV)   # unused entries hold no page
    at = 0
    for b, n in enumerate(n_pages):
        table[b, :n] = order[at:at + n]
        at += n
    shape = (sum(n_pages), hkv, page, d)
    s = dict(case=case, total=sum(new), max_q=max(new), max_kv=max(tot), table=table,
             kv_len=torch.tensor(tot, dtype=torch.int32, device=DEV),
             cu_q=torch.tensor([sum(new[:i]) for i in range(batch + 1)], dtype=torch.int32, device=DEV))
    normal = lambda *sh: torch.randn(sh, generator=g, device=DEV)
    total = sum(new)
    if case["op"] == "append":
        loud = torch.ones(d, device=DEV)
        loud[torch.randint(0, d, (3,), generator=g, device=DEV)] = 12.0      # channels with large activations
        row = lambda h, c: ((normal(total, h, d) * c).reshape(total, h * d)).to(torch.bfloat16)
        s.update(q=row(hq, loud), k=row(hkv, loud * 2), v=row(hkv, 1.0),
                 K=torch.zeros(shape, dtype=torch.bfloat16, device=DEV), V=torch.zeros(shape, dtype=torch.bfloat16, device=DEV),
                 q_out=torch.empty((total, hq * d), dtype=torch.bfloat16, device=DEV))
        s["gain_q"] = 1 + 0.1 * normal(d) if case["norm"] else None
        s["gain_k"] = 1 + 0.1 * normal(d) if case["norm"] else None
        i = torch.arange(total, device=DEV)
        b, p = i // case["new"], case["ctx"] + i % case["new"]
        s["pos"] = p.to(torch.int32)
        s["slots"] = table[b, p // page].to(torch.int64) * page + p % page
        return s
    if case["int8"]:
        s["K"] = (normal(*shape) * 32).round().clamp(-128, 127).to(torch.int8)
        s["V"] = (normal(*shape) * 32).round().clamp(-128, 127).to(torch.int8)
        s["k_scale"], s["v_scale"] = ((0.7 + 0.6 * torch.rand(hkv, generator=g, device=DEV)) / 32 for _ in range(2))
    else:
        s["K"], s["V"] = normal(*shape).to(torch.bfloat16), normal(*shape).to(torch.bfloat16)
        s["k_scale"] = s["v_scale"] = None
    if case["op"] == "evict":
        # a few keys hold most of the weight, as attention leaves it
        s["w"] = torch.exp(2.0 * normal(batch, hkv, max(tot)))
        keep = [-(-min(n, case["budget"]) // page) for n in tot]
        s["dst_table"] = torch.full((batch, -(-case["budget"] // page)), -1, dtype=torch.int32, device=DEV)
        order = torch.randperm(sum(keep), generator=g, device=DEV, dtype=torch.int32)
        at = 0
        for b, n in enumerate(keep):
            s["dst_table"][b, :n] = order[at:at + n]
            at += n
        s["dst_K"] = torch.zeros((sum(keep), hkv, page, d), dtype=s["K"].dtype, device=DEV)
        s["dst_V"] = torch.zeros_like(s["dst_K"])
        s["kept"] = torch.full((batch, hkv, case["budget"]), -1, dtype=torch.int32, device=DEV)
        s["w_out"] = torch.zeros((batch, hkv, case["budget"]), device=DEV)
        s["new_len"] = torch.zeros(batch, dtype=torch.int32, device=DEV)
        return s
    s["q"] = (normal(total, hq * d) * 1.2).to(torch.bfloat16)
    s["scale"] = 1.0 / math.sqrt(d)
    s["perm"] = None
    if case["aifs"]:
        s["perm"] = torch.tensor([p for n in new for p in _chunk_order(n)], dtype=torch.int32, device=DEV)
    if case["op"] == "attend":
        s["o"] = torch.empty((total, hq * d), dtype=torch.bfloat16, device=DEV)
        s["lse"] = torch.empty((total, hq), device=DEV)
    else:
        s["lse"] = _plain_scores(s)[1]            # the log-sum-exp that the attention of this step left
        s["w_in"] = 3.0 * torch.rand((batch, hkv, max(tot)), generator=g, device=DEV)
        s["w_out"] = torch.zeros((batch, hkv, max(tot)), device=DEV)
    return s


# ------------------------------------------------------------------------------------------------ plain form
def _plain_cached(s, name):
    """K or V of every sequence, padded to the longest: float32 [batch, hkv, keys, dim]."""
    pages = s[name][s["table"].clamp(min=0).long()].float()      # [batch, width, hkv, page, dim]
    if s[name].dtype == torch.int8:
        pages = pages * s[name.lower() + "_scale"][:, None, None]
    b, w, h, p, d = pages.shape
    return pages.permute(0, 2, 1, 3, 4).reshape(b, h, w * p, d)[:, :, :s["max_kv"]]


def _plain_rows(s):
    """(sequence, place in its chunk) of every new row."""
    r = torch.arange(s["total"], device=DEV)
    b = (r[:, None] >= s["cu_q"][None, 1:]).sum(1)
    return b, r - s["cu_q"][b].long()


def _plain_scores(s):
    """Masked scores [batch, hkv, group, rows, keys] and the log-sum-exp [total, hq], in float32."""
    c = s["case"]
    hq, hkv, d = c["hq"], c["hkv"], c["dim"]
    b, i = _plain_rows(s)
    q = torch.zeros((c["batch"], s["max_q"], hq, d), device=DEV)
    q[b, i] = s["q"].float().view(-1, hq, d)
    q = q.view(c["batch"], s["max_q"], hkv, hq // hkv, d).permute(0, 2, 3, 1, 4)
    k = _plain_cached(s, "K")
    sc = torch.matmul(q.reshape(c["batch"], hkv, -1, d), k.transpose(2, 3)) * s["scale"]
    sc = sc.view(c["batch"], hkv, hq // hkv, s["max_q"], -1)
    # a key of the cached context is visible to every new row; of the chunk, those that stood no later in the original order
    ctx = (s["kv_len"] - (s["cu_q"][1:] - s["cu_q"][:-1])).long()
    rank = torch.full((c["batch"], s["max_q"]), 2 ** 30, device=DEV)
    rank[b, i] = i if s["perm"] is None else s["perm"].long()
    key = torch.arange(s["max_kv"], device=DEV)[None] - ctx[:, None]                    # place in the chunk, < 0 in the context
    key_rank = torch.where(key < 0, -1, rank.gather(1, key.clamp(0, s["max_q"] - 1)))
    key_rank = torch.where(key >= s["max_q"], 2 ** 30, key_rank)
    seen = (key_rank[:, None] <= rank[:, :, None]) & (key_rank[:, None] < 2 ** 30)       # [batch, rows, keys]
    sc = torch.where(seen[:, None, None], sc, -math.inf)
    top = sc.amax(-1, keepdim=True)
    top = torch.where(top > -math.inf, top, 0.0)
    lse = (torch.log(torch.exp(sc - top).sum(-1)) + top[..., 0])                        # [batch, hkv, group, rows]
    return sc, lse.permute(0, 3, 1, 2)[b, i].reshape(-1, hq)


def _plain_attend(s):
    c = s["case"]
    sc, lse = _plain_scores(s)
    b, i = _plain_rows(s)
    top = sc.amax(-1, keepdim=True)
    p = torch.exp(sc - torch.where(top > -math.inf, top, 0.0))
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-30)
    o = torch.matmul(p.flatten(2, 3), _plain_cached(s, "V")).view(*p.shape[:4], c["dim"])
    return o.permute(0, 3, 1, 2, 4)[b, i].reshape(s["total"], -1).to(torch.bfloat16), lse


def _plain_weights(s):
    c = s["case"]
    sc, _ = _plain_scores(s)
    b, i = _plain_rows(s)
    lse = torch.full((c["batch"], s["max_q"], c["hq"]), math.inf, device=DEV)             # rows of the padding add nothing
    lse[b, i] = s["lse"]
    lse = lse.view(c["batch"], s["max_q"], c["hkv"], -1).permute(0, 2, 3, 1)
    got = torch.exp(sc - lse[..., None]).sum((2, 3))                                    # [batch, hkv, keys]
    ctx = s["kv_len"] - (s["cu_q"][1:] - s["cu_q"][:-1])
    at = torch.arange(s["max_kv"], device=DEV)[None, None]
    old = torch.where(at < ctx[:, None, None], s["w_in"], 0.0)                          # a new key has no weight yet
    return torch.where(at < s["kv_len"][:, None, None], old + got, s["w_out"])


def _plain_rotate(x, gain, s):
    """RMSNorm of every head (with a gain), then the rotary embedding: float32 [rows, heads, dim]."""
    c = s["case"]
    d = c["dim"]
    x = x.float().view(s["total"], -1, d)
    if gain is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * gain
    theta = 10000.0 ** (-2.0 * torch.arange(d // 2, device=DEV, dtype=torch.float64) / d)
    ang = s["pos"].double()[:, None] * theta
    cos, sin = torch.cos(ang).float()[:, None], torch.sin(ang).float()[:, None]
    a, b = (x[..., :d // 2], x[..., d // 2:]) if c["half"] else (x[..., 0::2], x[..., 1::2])
    u, v = a * cos - b * sin, a * sin + b * cos
    return torch.cat((u, v), -1) if c["half"] else torch.stack((u, v), -1).flatten(-2)


def _plain_append(s):
    c = s["case"]
    q = _plain_rotate(s["q"], s["gain_q"], s).reshape(s["total"], -1).to(torch.bfloat16)
    k = _plain_rotate(s["k"], s["gain_k"], s).to(torch.bfloat16)
    page, slot = s["slots"] // c["page"], s["slots"] % c["page"]
    s["K"][page, :, slot] = k
    s["V"][page, :, slot] = s["v"].view(s["total"], c["hkv"], c["dim"])
    return q, s["K"], s["V"]


def _plain_evict(s):
    c = s["case"]
    batch, hkv, budget = c["batch"], c["hkv"], c["budget"]
    at = torch.arange(s["max_kv"], device=DEV)
    n = s["kv_len"].long()[:, None, None]
    always = (at < c["first"]) | (at >= n - c["last"])
    w = torch.where(always, math.inf, s["w"])
    w = torch.where(at < n, w, -math.inf)
    rank = torch.sort(w, dim=-1, descending=True, stable=True).indices[..., :budget]    # ties: the lowest index first
    m = rank.shape[-1]
    count = n.clamp(max=budget)
    live = torch.arange(m, device=DEV) < count
    kept = torch.sort(torch.where(live, rank, 2 ** 30), dim=-1).values                  # in the order of the cache
    seq = torch.arange(batch, device=DEV)[:, None, None].expand(batch, hkv, m)
    head = torch.arange(hkv, device=DEV)[None, :, None].expand(batch, hkv, m)
    src = torch.where(live, kept, 0)
    to = torch.arange(m, device=DEV).expand(batch, hkv, m)
    from_page, from_slot = s["table"].long()[seq, src // c["page"]], src % c["page"]
    to_page, to_slot = s["dst_table"].long()[seq, to // c["page"]], to % c["page"]
    spare = s["dst_K"].shape[0]                                                          # where rows past the count go
    for name in ("K", "V"):
        wide = torch.cat((s["dst_" + name], s["dst_" + name][:1]))
        wide[torch.where(live, to_page, spare), head, to_slot] = s[name][from_page, head, from_slot]
        s["dst_" + name].copy_(wide[:spare])
    s["kept"][..., :m] = torch.where(live, kept, s["kept"][..., :m].long()).int()
    s["w_out"][..., :m] = torch.where(live, s["w"].gather(2, src), s["w_out"][..., :m])
    s["new_len"].copy_(count.flatten())
    return s["dst_K"], s["dst_V"], s["kept"], s["w_out"], s["new_len"]


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    op = s["case"]["op"]
    if not own:
        return {"append": _plain_append, "attend": _plain_attend, "weights": _plain_weights, "evict": _plain_evict}[op](s)
    from paper_2502_00425_b200 import binding as B
    c = s["case"]
    if "cache" not in s:   # what a serving program keeps: the cache's handle and the attention's workspace
        s["cache"] = B.KVCache(s["K"], s["V"], s.get("k_scale"), s.get("v_scale"))
        if op == "attend":
            s["ws"] = B.new_kv_attention_workspace(c["batch"], s["total"], s["max_q"], s["table"].shape[1], c["hq"], s["cache"])
        if op == "evict":
            s["dst"] = B.KVCache(s["dst_K"], s["dst_V"], s.get("k_scale"), s.get("v_scale"))
    if op == "append":
        B.mq_qk_norm_rope(s["q"], s["k"], s["pos"], c["hq"], c["hkv"], s["q_out"], gain_q=s["gain_q"], gain_k=s["gain_k"],
                          half=c["half"], v=s["v"], cache=s["cache"], slots=s["slots"])
        return s["q_out"], s["K"], s["V"]
    if op == "attend":
        B.mq_kv_attention(s["q"], s["cu_q"], s["kv_len"], s["table"], s["cache"], c["hq"], s["max_q"], s["o"], s["ws"],
                          lse=s["lse"], perm=s["perm"], scale=s["scale"])
        return s["o"], s["lse"]
    if op == "weights":
        B.mq_kv_weights(s["q"], s["cu_q"], s["kv_len"], s["table"], s["cache"], c["hq"], s["max_q"], s["lse"], s["w_out"],
                        w_in=s["w_in"], perm=s["perm"], scale=s["scale"])
        return s["w_out"]
    B.mq_kv_evict(s["cache"], s["table"], s["kv_len"], s["w"], c["budget"], c["first"], c["last"], s["dst"], s["dst_table"],
                  s["kept"], s["new_len"], w_out=s["w_out"])
    return s["dst_K"], s["dst_V"], s["kept"], s["w_out"], s["new_len"]


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def _exact_keys(s, name, b, h, n):
    page = s["case"]["page"]
    j = torch.arange(n, device=DEV)
    rows = s[name][s["table"][b, j // page].long(), h, j % page].double()
    return rows * s[name.lower() + "_scale"][h].double() if s[name].dtype == torch.int8 else rows


def _exact_softmax(s, b, h, head, n_new, n_all, start):
    """Scores of one query head over its keys, -inf where a row may not look."""
    d = s["case"]["dim"]
    q = s["q"][start:start + n_new, head * d:(head + 1) * d].double()
    sc = q @ _exact_keys(s, "K", b, h, n_all).T * s["scale"]
    own_rank = torch.arange(n_new, device=DEV) if s["perm"] is None else s["perm"][start:start + n_new].long()
    sc[:, n_all - n_new:].masked_fill_(own_rank[None, :] > own_rank[:, None], -math.inf)
    return sc


def exact(case, seed):
    s = prepare(case, seed)
    new, tot = _lens(case)
    hq, hkv, d, page = case["hq"], case["hkv"], case["dim"], case["page"]
    total = sum(new)
    if case["op"] == "append":
        i = torch.arange(d, device=DEV)
        pair = i % (d // 2) if case["half"] else i // 2
        ang = s["pos"].double()[:, None] * torch.pow(torch.tensor(10000.0, dtype=torch.float64, device=DEV), -2.0 * pair.double() / d)
        mate = (i + d // 2) % d if case["half"] else i ^ 1
        sign = torch.where((i < d // 2) if case["half"] else (i % 2 == 0), -1.0, 1.0).double()

        def rotated(x, heads, gain):
            x = x.double().view(total, heads, d)
            if gain is not None:
                x = x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / d + 1e-6) * gain.double()
            return x * ang.cos()[:, None] + sign * x[..., mate] * ang.sin()[:, None]

        K, V = s["K"].double(), s["V"].double()
        k, v = rotated(s["k"], hkv, s["gain_k"]), s["v"].double().view(total, hkv, d)
        flat = lambda c: c.permute(0, 2, 1, 3).reshape(-1, hkv, d)
        out = []
        for c, rows in ((K, k), (V, v)):
            f = flat(c).clone()
            f[s["slots"]] = rows
            out.append(f.view(c.shape[0], page, hkv, d).permute(0, 2, 1, 3).contiguous())
        return rotated(s["q"], hq, s["gain_q"]).reshape(total, hq * d), out[0], out[1]
    if case["op"] == "evict":
        K, V, w_out = s["dst_K"].double(), s["dst_V"].double(), s["w_out"].double()
        for b, n in enumerate(tot):
            for h in range(hkv):
                w = s["w"][b, h, :n].double()
                w[:case["first"]] = math.inf
                w[max(0, n - case["last"]):] = math.inf
                keep = torch.argsort(-w, stable=True)[:case["budget"]].sort().values
                j = torch.arange(keep.numel(), device=DEV)
                to = s["dst_table"][b, j // page].long()
                for c, name in ((K, "K"), (V, "V")):
                    c[to, h, j % page] = s[name][s["table"][b, keep // page].long(), h, keep % page].double()
                w_out[b, h, :keep.numel()] = s["w"][b, h, keep].double()
        return K, V, None, w_out, None
    group = hq // hkv
    o = torch.zeros((total, hq * d), dtype=torch.float64, device=DEV)
    lse = torch.zeros((total, hq), dtype=torch.float64, device=DEV)
    w = s["w_out"].double() if case["op"] == "weights" else None
    start = 0
    for b, (n_new, n_all) in enumerate(zip(new, tot)):
        for h in range(hkv):
            if w is not None:
                w[b, h, :n_all] = s["w_in"][b, h, :n_all].double()
                w[b, h, n_all - n_new:n_all] = 0.0
            for head in range(h * group, (h + 1) * group):
                sc = _exact_softmax(s, b, h, head, n_new, n_all, start)
                if w is not None:
                    w[b, h, :n_all] += torch.exp(sc - s["lse"][start:start + n_new, head].double()[:, None]).sum(0)
                    continue
                l = torch.logsumexp(sc, -1)
                lse[start:start + n_new, head] = l
                o[start:start + n_new, head * d:(head + 1) * d] = torch.exp(sc - l[:, None]) @ _exact_keys(s, "V", b, h, n_all)
        start += n_new
    return w if w is not None else (o, lse)
