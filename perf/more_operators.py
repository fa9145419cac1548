"""What a serving step needs around the paged cache, for measurement.

  plan     pages, cumulative row counts, cache slots and positions of a step, from the lengths that the sequences ask for;
  rotary   RMSNorm of every query and key head, the rotary embedding of a part of the head or scaled for a long context, and
           the store of K and V into the cache's pages;
  shared   grouped-query attention over the paged cache for sequences that share a long prefix, which is read once per group;
  sample   the next tokens from logits: temperature, top-k, top-p and min-p, from given random numbers.

`own` false: the plain form, elementary torch operations in 32 bits (64 for angles and for the sums that a border is found in).
`own` true: the library's entry points.  `exact` is the definition in 64 bits, one row, sequence or head at a time.
"""
import math

import torch

own = False
DEV = "cuda"


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # a speculative step of a decoding batch (and its undoing): latency
        dict(name="plan decode 256", op="plan", batch=256, new_lo=1, new_hi=5, ctx_lo=100, ctx_hi=6000, page=64, done=0.1),
        # a batch of prompts admitted at once, some of their sequences in place of finished ones
        dict(name="plan prompts 64", op="plan", batch=64, new_lo=200, new_hi=3360, ctx_lo=1, ctx_hi=3000, page=16, done=0.5),
        # one decode step of 32 sequences far behind the context that the rotary embedding was made for
        dict(name="rotary long decode 32", op="rotary", batch=32, new=1, ctx=70000, hq=28, hkv=4, dim=128, page=64, norm=False, half=True,
             rot=128, factor=4.0, original=32768),
        # the prompts of the 4 x 2432-token batch, half of every head rotated
        dict(name="rotary part prompt 9728", op="rotary", batch=4, new=2432, ctx=0, hq=32, hkv=8, dim=128, page=128, norm=True, half=True,
             rot=64, factor=1.0, original=0),
        # 32 questions about one prompt of three images, each some tokens into its answer
        dict(name="shared 32 over 3360", op="shared", batch=32, groups=1, prefix=3360, new_lo=1, new_hi=1, own_lo=16, own_hi=400, hq=28,
             hkv=4, dim=128, page=64, int8=False, aifs=False),
        # four image prompts with 16 answers each, on an 8-bit cache
        dict(name="shared 4 x 16 int8", op="shared", batch=64, groups=4, prefix=2432, new_lo=1, new_hi=1, own_lo=30, own_hi=900, hq=32,
             hkv=8, dim=128, page=64, int8=True, aifs=False),
        # follow-up questions with an image in each, one document in front of them
        dict(name="shared turns aifs", op="shared", batch=6, groups=1, prefix=8192, new_lo=5, new_hi=60, own_lo=40, own_hi=600, hq=32,
             hkv=8, dim=128, page=16, int8=False, aifs=True),
        # the largest: many answers behind a long document
        dict(name="shared 128 over 32768", op="shared", batch=128, groups=1, prefix=32768, new_lo=1, new_hi=1, own_lo=64, own_hi=2048,
             hq=32, hkv=8, dim=128, page=128, int8=False, aifs=False),
        # one chat's next token: latency
        dict(name="sample 1 x 131072", op="sample", batch=1, vocab=131072, pitch=131072, f32=True, mode="usual"),
        # a batch whose rows ask for different things: greedy, unfiltered, each filter alone, all of them, masked rows
        dict(name="sample 64 x 131072 mixed", op="sample", batch=64, vocab=131072, pitch=131072, f32=True, mode="mixed"),
        # bf16 logits of a padded head, an odd vocabulary, top-p alone
        dict(name="sample 32 x 50001 bf16", op="sample", batch=32, vocab=50001, pitch=50048, f32=False, mode="top_p"),
        # a large batch, everything on
        dict(name="sample 256 x 150001", op="sample", batch=256, vocab=150001, pitch=150016, f32=True, mode="usual"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["plan", "rotary", "shared", "shared", "shared", "sample", "sample", "sample"])
    hq, hkv = rng.choice([(28, 4), (32, 8)])
    dim, page = rng.choice([128, 128, 64]), rng.choice([16, 32, 64, 128])
    if op == "plan":
        batch = _log_int(rng, 1, 1024)
        lo, hi = sorted((_log_int(rng, 1, 4096), _log_int(rng, 1, 4096)))
        top = max(1, 131072 // batch)
        new_lo, new_hi = sorted((_log_int(rng, 1, min(top, 8192)), _log_int(rng, 1, min(top, 8192))))
        return dict(op=op, batch=batch, new_lo=new_lo, new_hi=new_hi, ctx_lo=lo, ctx_hi=hi, page=page, done=rng.choice([0.0, 0.1, 0.5]))
    if op == "rotary":
        batch = _log_int(rng, 1, 64)
        factor = rng.choice([1.0, 2.0, 4.0, 8.0])
        return dict(op=op, batch=batch, new=_log_int(rng, 1, max(1, 9728 // batch)), ctx=rng.randrange(0, 100000), hq=hq, hkv=hkv, dim=dim,
                    page=page, norm=rng.random() < 0.5, half=rng.random() < 0.5, rot=8 * rng.randrange(1, dim // 8 + 1), factor=factor,
                    original=rng.choice([0, 4096, 32768]) if factor > 1 else 0)
    if op == "shared":
        batch = _log_int(rng, 2, 128)
        new_hi = rng.choice([1, 1, 1, 3, 40])
        lo, hi = sorted((_log_int(rng, 1, 2048), _log_int(rng, 16, 2048)))
        return dict(op=op, batch=batch, groups=rng.randrange(1, 1 + min(8, batch // 2)), prefix=_log_int(rng, 40, 16384), new_lo=1,
                    new_hi=min(new_hi, max(1, 512 // batch)), own_lo=lo, own_hi=hi, hq=hq, hkv=hkv, dim=dim, page=page,
                    int8=rng.random() < 0.35, aifs=new_hi > 3 and rng.random() < 0.5)
    vocab = _log_int(rng, 1000, 150001)
    return dict(op=op, batch=_log_int(rng, 1, 256), vocab=vocab, pitch=vocab + rng.choice([0, 0, 1, 15, 64]), f32=rng.random() < 0.5,
                mode=rng.choice(["mixed", "usual", "top_p", "top_k", "plain"]))


def _spread(lo, hi, n, phase):
    """n lengths from lo to hi, evenly over their logarithm, in a mixed-up order; both ends are among them when n > 1."""
    if n == 1:
        return [hi]
    vals = [int(round(math.exp(math.log(lo) + (math.log(hi) - math.log(lo)) * i / (n - 1)))) for i in range(n)]
    step = next(s for s in range(n // 2 + 1 + phase, 4 * n) if math.gcd(s, n) == 1)
    return [vals[(i * step + phase) % n] for i in range(n)]


def _plan_lens(case):
    """(new rows, keys cached, keys kept) of every sequence: one in 1 / done has finished, and every second of those begins again."""
    n = case["batch"]
    new, ctx = _spread(case["new_lo"], case["new_hi"], n, 0), _spread(case["ctx_lo"], case["ctx_hi"], n, 1)
    every = round(1 / case["done"]) if case["done"] else 0
    over = [bool(every) and b % every == every - 1 for b in range(n)]
    new = [0 if over[b] and (b // every) % 2 == 0 else new[b] for b in range(n)]
    return new, ctx, [0 if over[b] else ctx[b] for b in range(n)]


def _shared_lens(case):
    """(first sequence of its group, new rows, keys of its own with them) of every sequence, and the keys of a group's whole shared pages."""
    n, g = case["batch"], case["groups"]
    first = [-(-n * (b * g // n) // g) for b in range(n)]
    new, mine = _spread(case["new_lo"], case["new_hi"], n, 0), _spread(case["own_lo"], case["own_hi"], n, 1)
    shared = case["prefix"] // case["page"] * case["page"]
    return first, new, [case["prefix"] - shared + a + b for a, b in zip(new, mine)], shared


def work(case):
    op = case["op"]
    if op == "plan":
        new, ctx, keep = _plan_lens(case)
        pages = sum(abs(-(-(k + a) // case["page"]) - -(-c // case["page"])) for a, c, k in zip(new, ctx, keep))
        # two calls: lengths in and out, a slot and a position per row, a table entry and a free page per page that moves
        return {"bytes": 12 * sum(new) + 2 * (24 * case["batch"] + 8 * pages), "flops": 4 * sum(new)}
    if op == "rotary":
        t, hq, hkv, d = case["batch"] * case["new"], case["hq"], case["hkv"], case["dim"]
        return {"bytes": t * (2 * (hq + 2 * hkv) * d * 2 + 12), "flops": t * (hq + hkv) * (6 * case["rot"] + (4 * d if case["norm"] else 0))}
    if op == "shared":
        first, new, mine, shared = _shared_lens(case)
        hq, hkv, d, es = case["hq"], case["hkv"], case["dim"], 1 if case["int8"] else 2
        keys = sum(mine) + shared * len(set(first))
        pairs = sum(n * (shared + k - n) + n * (n + 1) // 2 for n, k in zip(new, mine))
        return {"bytes": sum(new) * hq * (4 * d + 4) + keys * hkv * 2 * d * es, "flops": 4 * d * hq * pairs}
    n = case["batch"] * case["vocab"]
    return {"bytes": n * (4 if case["f32"] else 2) + 32 * case["batch"], "flops": 8 * n}


# ------------------------------------------------------------------------------------------------ inputs
def _prepare_plan(case, g):
    new, ctx, keep = _plan_lens(case)
    n, page = case["batch"], case["page"]
    pages = [-(-c // page) for c in ctx]
    total = sum(pages) + sum(-(-a // page) + 1 for a in new)
    width = -(-max(max(k + a, c) for a, c, k in zip(new, ctx, keep)) // page) + 1
    order = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
    table = torch.full((n, width), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, m in enumerate(pages):
        table[b, :m] = order[at:at + m]
        at += m
    free = torch.full((total,), -1, dtype=torch.int32, device=DEV)
    free[:total - at] = order[at:]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
    rows = sum(new) + 3                                                          # (a graph's row count is a bound)
    behind = torch.randint(0, 50, (n,), generator=g, device=DEV, dtype=torch.int32)  # tokens that were evicted earlier
    s = dict(case=case, kv_len=ints(ctx), table=table, free=free, n_free=ints([total - at]), new=ints(new), keep=ints(keep), rows=rows,
             seen=ints(ctx) + torch.where(ints(keep) > 0, behind, 0),
             cu_q=torch.zeros(n + 1, dtype=torch.int32, device=DEV), slots=torch.zeros(rows, dtype=torch.int64, device=DEV),
             pos=torch.zeros(rows, dtype=torch.int32, device=DEV), status=torch.zeros(2, dtype=torch.int32, device=DEV))
    # the step back: what the sequences had, from what they have then
    after = [k + a for a, k in zip(new, keep)]
    s["back_keep"] = ints([min(c, k) for c, k in zip(ctx, keep)])
    s["back_new"] = ints([c - min(c, k) for c, k in zip(ctx, keep)])
    s["back_rows"] = max(1, sum(c - min(c, k) for c, k in zip(ctx, keep)))
    s["back"] = [torch.zeros(n + 1, dtype=torch.int32, device=DEV), torch.zeros(s["back_rows"], dtype=torch.int64, device=DEV),
                 torch.zeros(s["back_rows"], dtype=torch.int32, device=DEV)]
    assert max(after) <= width * page
    return s


def _prepare_rotary(case, g):
    hq, hkv, d, page, batch = case["hq"], case["hkv"], case["dim"], case["page"], case["batch"]
    total = batch * case["new"]
    normal = lambda *sh: torch.randn(sh, generator=g, device=DEV)
    loud = torch.ones(d, device=DEV)
    loud[torch.randint(0, d, (3,), generator=g, device=DEV)] = 12.0              # channels with large activations
    row = lambda h, c: ((normal(total, h, d) * c).reshape(total, h * d)).to(torch.bfloat16)
    s = dict(case=case, q=row(hq, loud), k=row(hkv, loud * 2), v=row(hkv, 1.0), q_out=torch.empty((total, hq * d), dtype=torch.bfloat16, device=DEV))
    n_pages = -(-total // page)
    s["K"], s["V"] = (torch.zeros((n_pages, hkv, page, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    s["slots"] = torch.randperm(n_pages * page, generator=g, device=DEV)[:total].contiguous() if case["new"] == 1 else torch.arange(total, device=DEV)
    s["pos"] = (case["ctx"] + torch.arange(total, device=DEV) % case["new"] + 37 * (torch.arange(total, device=DEV) // case["new"])).to(torch.int32)
    s["gain_q"] = 1 + 0.1 * normal(d) if case["norm"] else None
    s["gain_k"] = 1 + 0.1 * normal(d) if case["norm"] else None
    s["amp"] = 0.1 * math.log(case["factor"]) + 1.0 if case["original"] else 1.0
    return s


def _chunk_order(n):
    """AIFS order of a chunk [text][image][text]: its visual tokens first, then its text tokens."""
    a, b = n // 5, n - n // 4
    return list(range(a, b)) + list(range(a)) + list(range(b, n))


def _prepare_shared(case, g):
    first, new, mine, shared = _shared_lens(case)
    hq, hkv, d, page, n = case["hq"], case["hkv"], case["dim"], case["page"], case["batch"]
    n_shared, n_mine = shared // page, [-(-m // page) for m in mine]
    n_pages = n_shared * len(set(first)) + sum(n_mine)
    order = torch.randperm(n_pages, generator=g, device=DEV, dtype=torch.int32)
    table = torch.full((n, n_shared + max(n_mine) + 1), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b in range(n):
        if first[b] == b:
            table[b, :n_shared] = order[at:at + n_shared]
            at += n_shared
        else:
            table[b, :n_shared] = table[first[b], :n_shared]
        table[b, n_shared:n_shared + n_mine[b]] = order[at:at + n_mine[b]]
        at += n_mine[b]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
    normal = lambda *sh: torch.randn(sh, generator=g, device=DEV)
    total, shape = sum(new), (n_pages, hkv, page, d)
    s = dict(case=case, total=total, max_q=max(new), table=table, kv_len=ints([shared + m for m in mine]),
             cu_q=ints([sum(new[:i]) for i in range(n + 1)]), leader=ints(first), shared_len=ints([shared] * n))
    if case["int8"]:
        s["K"], s["V"] = ((normal(*shape) * 32).round().clamp(-128, 127).to(torch.int8) for _ in range(2))
        s["k_scale"], s["v_scale"] = ((0.7 + 0.6 * torch.rand(hkv, generator=g, device=DEV)) / 32 for _ in range(2))
    else:
        s["K"], s["V"] = normal(*shape).to(torch.bfloat16), normal(*shape).to(torch.bfloat16)
        s["k_scale"] = s["v_scale"] = None
    s["q"] = (normal(total, hq * d) * 1.2).to(torch.bfloat16)
    s["scale"] = 1.0 / math.sqrt(d)
    s["perm"] = ints([p for m in new for p in _chunk_order(m)]) if case["aifs"] else None
    s["o"] = torch.empty((total, hq * d), dtype=torch.bfloat16, device=DEV)
    s["lse"] = torch.empty((total, hq), device=DEV)
    return s


def _prepare_sample(case, g):
    n, v, mode = case["batch"], case["vocab"], case["mode"]
    normal = lambda *sh: torch.randn(sh, generator=g, device=DEV)
    # a bulk of unlikely tokens and some dozens that stand out, sharper in some rows than in others
    x = 2.2 * normal(n, case["pitch"])
    at = torch.randint(0, v, (n, min(v, 48)), generator=g, device=DEV)
    x.scatter_add_(1, at, 9.0 + 3.0 * normal(n, at.shape[1]))
    x *= 0.6 + torch.rand((n, 1), generator=g, device=DEV)
    i = torch.arange(n, device=DEV)
    kind = i % 8 if mode == "mixed" else torch.full_like(i, {"usual": 6, "top_p": 2, "top_k": 3, "plain": 1}[mode])
    if mode == "mixed":                                                          # a grammar allows every third token only
        x[(kind == 7)[:, None] & (torch.arange(case["pitch"], device=DEV) % 3 > 0)[None]] = -math.inf
    f = lambda on, lo, hi, off: torch.where(on, lo + (hi - lo) * torch.rand(n, generator=g, device=DEV), off)
    k = torch.randint(1, 200, (n,), generator=g, device=DEV)
    k = torch.where(i % 5 == 4, k * 40, k)                                       # some ask for thousands
    s = dict(case=case, x=x.float() if case["f32"] else x.to(torch.bfloat16), temperature=f(kind > 0, 0.5, 1.3, 0.0),
             top_p=f((kind == 2) | (kind >= 5), 0.7, 0.98, 1.0), min_p=f((kind == 4) | (kind == 5) | (kind == 6) & (i % 2 == 1), 0.005, 0.1, 0.0),
             top_k=torch.where((kind == 3) | (kind >= 6), k, 0).to(torch.int32), u=torch.rand(n, generator=g, device=DEV))
    s["x"] = s["x"][:, :v]
    s["token"] = torch.empty(n, dtype=torch.int32, device=DEV)
    s["logp"] = torch.empty(n, device=DEV)
    s["kept"] = torch.empty(n, dtype=torch.int32, device=DEV)
    return s


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return {"plan": _prepare_plan, "rotary": _prepare_rotary, "shared": _prepare_shared, "sample": _prepare_sample}[case["op"]](case, g)


# ------------------------------------------------------------------------------------------------ plain form
def _plain_plan_call(s, new, keep, cu_q, slots, pos):
    page, rows = s["case"]["page"], slots.shape[0]
    table, free = s["table"], s["free"]
    old = s["kv_len"].long()
    keep, new = torch.minimum(keep.long(), old), new.long()
    p0, p2 = (old + page - 1) // page, (keep + new + page - 1) // page
    at = torch.arange(table.shape[1], device=DEV)[None]
    freed, taken = (at >= p2[:, None]) & (at < p0[:, None]), (at >= p0[:, None]) & (at < p2[:, None])
    rank = lambda m: torch.cumsum(m.flatten().long(), 0).view_as(m) - 1          # in the order of sequence and page
    top = s["n_free"].long() + freed.sum()
    stack = torch.cat((free, free[:1]))                                          # (a place for what moves nowhere)
    stack[torch.where(freed, top - 1 - rank(freed), free.shape[0])] = table
    got = stack[(top - 1 - rank(taken)).clamp(min=0)]
    table.copy_(torch.where(taken, got, table))
    free.copy_(stack[:-1])
    s["n_free"].copy_(top - taken.sum())
    s["kv_len"].copy_(keep + new)
    s["seen"].copy_(torch.where(keep > 0, s["seen"] - (old - keep), 0) + new)
    cu = torch.cat((torch.zeros(1, dtype=torch.long, device=DEV), torch.cumsum(new, 0)))
    cu_q.copy_(cu)
    r = torch.arange(rows, device=DEV)
    b = (torch.searchsorted(cu, r, right=True) - 1).clamp(max=new.shape[0] - 1)
    j = keep[b] + r - cu[b]
    live = r < cu[-1]
    slots.copy_(torch.where(live, table[b, torch.where(live, j // page, 0)].long() * page + j % page, -1))
    pos.copy_(torch.where(live, s["seen"][b] - (cu[b + 1] - r), 0))


def _plain_plan(s):
    _plain_plan_call(s, s["new"], s["keep"], s["cu_q"], s["slots"], s["pos"])
    _plain_plan_call(s, s["back_new"], s["back_keep"], *s["back"])


def _theta(c):
    """Radians per position of every rotated pair, in 64 bits."""
    r = c["rot"]
    theta = 10000.0 ** (-2.0 * torch.arange(r // 2, device=DEV, dtype=torch.float64) / r)
    if not c["original"]:
        return theta / c["factor"]
    turns = c["original"] * theta / (2 * math.pi)
    ramp = ((turns - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
    return theta * (ramp + (1 - ramp) / c["factor"])


def _plain_rotate(x, gain, s):
    c = s["case"]
    d, r = c["dim"], c["rot"]
    x = x.float().view(x.shape[0], -1, d)
    if gain is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * gain
    ang = s["pos"].double()[:, None] * _theta(c)
    cos, sin = (torch.cos(ang) * s["amp"]).float()[:, None], (torch.sin(ang) * s["amp"]).float()[:, None]
    a, b = (x[..., :r // 2], x[..., r // 2:r]) if c["half"] else (x[..., 0:r:2], x[..., 1:r:2])
    u, v = a * cos - b * sin, a * sin + b * cos
    return torch.cat((torch.cat((u, v), -1) if c["half"] else torch.stack((u, v), -1).flatten(-2), x[..., r:]), -1)


def _plain_rotary(s):
    c = s["case"]
    q = _plain_rotate(s["q"], s["gain_q"], s).reshape(s["q"].shape).to(torch.bfloat16)
    page, slot = s["slots"] // c["page"], s["slots"] % c["page"]
    s["K"][page, :, slot] = _plain_rotate(s["k"], s["gain_k"], s).to(torch.bfloat16)
    s["V"][page, :, slot] = s["v"].view(-1, c["hkv"], c["dim"])
    return q, s["K"], s["V"]


def _plain_keys(s, name, pages):
    """K or V of lists of pages [n, width]: float32 [n, heads, keys, dim]."""
    x = s[name][pages.clamp(min=0).long()].float()
    if s[name].dtype == torch.int8:
        x = x * s[name.lower() + "_scale"][:, None, None]
    n, w, h, p, d = x.shape
    return x.permute(0, 2, 1, 3, 4).reshape(n, h, w * p, d)


def _plain_shared(s):
    c = s["case"]
    first, new, mine, shared = _shared_lens(c)                                   # (what the host knows of its batch)
    hq, hkv, d, page, n_shared = c["hq"], c["hkv"], c["dim"], c["page"], shared // c["page"]
    out, lses, row = [], [], 0
    for a in sorted(set(first)):
        e = a + first.count(a)
        m, wide, rows = e - a, max(mine[a:e]), max(new[a:e])
        lens, n_new = s["kv_len"][a:e] - shared, s["cu_q"][a + 1:e + 1] - s["cu_q"][a:e]
        i = torch.arange(sum(new[a:e]), device=DEV)
        b = ((row + i)[:, None] >= s["cu_q"][None, a + 1:e + 1]).sum(1)
        j = row + i - s["cu_q"][a:e][b]
        q = torch.zeros((m, rows, hq, d), device=DEV)
        q[b, j] = s["q"][row:row + i.shape[0]].float().view(-1, hq, d)
        q = q.view(m, rows, hkv, hq // hkv, d).permute(2, 0, 3, 1, 4)            # [heads, sequences, group, rows, dim]
        rank = torch.full((m, rows), 2 ** 30, device=DEV)
        rank[b, j] = j if s["perm"] is None else s["perm"][row:row + i.shape[0]].long()
        k0, v0 = (_plain_keys(s, x, s["table"][a:a + 1, :n_shared])[0] for x in ("K", "V"))
        k1, v1 = (_plain_keys(s, x, s["table"][a:e, n_shared:])[:, :, :wide].transpose(0, 1) for x in ("K", "V"))
        s0 = torch.matmul(q.reshape(hkv, -1, d), k0.transpose(1, 2)).view(hkv, m, hq // hkv, rows, -1) * s["scale"]
        s1 = torch.matmul(q.flatten(2, 3), k1.transpose(2, 3)).view(hkv, m, hq // hkv, rows, -1) * s["scale"]
        key = torch.arange(wide, device=DEV)[None] - (lens - n_new)[:, None]     # place in the chunk, < 0 before it
        key_rank = torch.where(key < 0, -1, rank.gather(1, key.clamp(0, rows - 1)))
        key_rank = torch.where(key >= n_new[:, None], 2 ** 30, key_rank)
        seen = (key_rank[:, None] <= rank[:, :, None]) & (key_rank[:, None] < 2 ** 30)
        s1 = torch.where(seen[None, :, None], s1, -math.inf)
        top = torch.maximum(s0.amax(-1, keepdim=True) if shared else torch.full_like(s1[..., :1], -math.inf), s1.amax(-1, keepdim=True))
        top = torch.where(top > -math.inf, top, 0.0)
        e0, e1 = torch.exp(s0 - top), torch.exp(s1 - top)
        z = e0.sum(-1, keepdim=True) + e1.sum(-1, keepdim=True)
        o = torch.matmul(e0.view(hkv, -1, e0.shape[-1]), v0).view(*e0.shape[:4], d) + torch.matmul(e1.flatten(2, 3), v1).view(*e1.shape[:4], d)
        o, lse = o / z.clamp(min=1e-30), torch.log(z[..., 0]) + top[..., 0]
        out.append(o.permute(1, 3, 0, 2, 4)[b, j].reshape(-1, hq * d))
        lses.append(lse.permute(1, 3, 0, 2)[b, j].reshape(-1, hq))
        row += i.shape[0]
    return torch.cat(out).to(torch.bfloat16), torch.cat(lses)


def _plain_sample(s):
    """Weights and their sums in 64 bits: a border falls between two tokens of a hundred thousand."""
    x = s["x"]
    x = torch.where(torch.isnan(x), -math.inf, x)
    n, v = x.shape
    t = s["temperature"].double()[:, None]
    sorted_x, order = torch.sort(x, dim=1, descending=True, stable=True)         # equal logits: the lowest index first
    top = sorted_x[:, :1].double()
    gap = torch.where(sorted_x == sorted_x[:, :1], 0.0, sorted_x.double() - top)
    w = torch.where(sorted_x > -math.inf, torch.exp(gap / t.clamp(min=1e-300)), 0.0)
    rank = torch.arange(v, device=DEV)[None]
    k = s["top_k"].long()[:, None]
    keep = (sorted_x > -math.inf) & ((k <= 0) | (rank < k))
    w = torch.where(keep, w, 0.0)
    p = s["top_p"].double()[:, None]
    before = torch.cumsum(w, 1) - w
    keep &= (p >= 1.0) | (before < p * w.sum(1, keepdim=True))
    keep &= w >= s["min_p"].double()[:, None]
    keep[:, 0] = sorted_x[:, 0] > -math.inf
    keep &= (t > 0) | (rank == 0)
    w = torch.zeros_like(w).scatter_(1, order, torch.where(keep, w, 0.0))        # back in the order of the vocabulary
    run_sum = torch.cumsum(w, 1)
    total = run_sum[:, -1:]
    token = (run_sum <= s["u"].double()[:, None] * total).sum(1, keepdim=True).clamp(max=v - 1)
    logp = torch.log(w.gather(1, token) / total)[:, 0].float()
    return token[:, 0].int(), logp, keep.sum(1).int()


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    c, op = s["case"], s["case"]["op"]
    if not own:
        if op == "plan":
            _plain_plan(s)
        else:
            return {"rotary": _plain_rotary, "shared": _plain_shared, "sample": _plain_sample}[op](s)
    else:
        from paper_2502_00425_b200 import binding as B
        if op == "plan":
            if "state" not in s:
                s["state"] = B.KVState(s["kv_len"], s["seen"], s["table"], s["free"], s["n_free"], c["page"])
            B.mq_kv_plan(s["state"], s["new"], s["cu_q"], s["slots"], s["pos"], s["status"], keep=s["keep"])
            B.mq_kv_plan(s["state"], s["back_new"], *s["back"], s["status"], keep=s["back_keep"])
        elif op == "sample":
            B.mq_sample(s["x"], s["temperature"], s["u"], s["token"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"], logp=s["logp"],
                        kept=s["kept"])
            return s["token"], s["logp"], s["kept"]
        else:
            if "cache" not in s:   # what a serving program keeps: the cache's handle, the embedding's frequencies, the workspace
                s["cache"] = B.KVCache(s["K"], s["V"], s.get("k_scale"), s.get("v_scale"))
                if op == "rotary":
                    s["rope"] = B.Rope(c["rot"], half=c["half"], factor=c["factor"], original=c["original"], amp=s["amp"])
                else:
                    s["ws"] = B.new_kv_attention_shared_workspace(c["batch"], s["total"], s["max_q"], s["table"].shape[1], c["hq"], s["cache"])
            if op == "rotary":
                B.mq_qk_norm_rope_scaled(s["q"], s["k"], s["pos"], c["hq"], c["hkv"], s["q_out"], s["rope"], gain_q=s["gain_q"],
                                         gain_k=s["gain_k"], v=s["v"], cache=s["cache"], slots=s["slots"])
                return s["q_out"], s["K"], s["V"]
            B.mq_kv_attention_shared(s["q"], s["cu_q"], s["kv_len"], s["table"], s["leader"], s["shared_len"], s["cache"], c["hq"], s["max_q"],
                                     s["o"], s["ws"], lse=s["lse"], perm=s["perm"], scale=s["scale"])
            return s["o"], s["lse"]
    return (s["cu_q"], s["slots"], s["pos"], *s["back"], s["kv_len"], s["seen"], s["table"], s["free"], s["n_free"])


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def _exact_rotary(s):
    c = s["case"]
    d, r, half = c["dim"], c["rot"], c["half"]
    q, k = (x.double().view(x.shape[0], -1, d) for x in (s["q"], s["k"]))
    out = []
    for x, gain in ((q, s["gain_q"]), (k, s["gain_k"])):
        if gain is not None:
            x = x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / d + 1e-6) * gain.double()
        y = x.clone()
        for i in range(r // 2):
            theta = math.pow(10000.0, -2.0 * i / r)
            if c["original"]:
                share = min(1.0, max(0.0, (c["original"] / (2 * math.pi / theta) - 1.0) / 31.0))
                theta = share * theta + (1.0 - share) * theta / c["factor"]
            else:
                theta /= c["factor"]
            z = torch.polar(torch.full_like(s["pos"], 1, dtype=torch.float64) * s["amp"], s["pos"].double() * theta)[:, None]
            a, b = (i, i + r // 2) if half else (2 * i, 2 * i + 1)
            turned = torch.complex(x[..., a], x[..., b]) * z
            y[..., a], y[..., b] = turned.real, turned.imag
        out.append(y)
    pools = []
    for pool, rows in ((s["K"], out[1]), (s["V"], s["v"].double().view(-1, c["hkv"], d))):
        flat = pool.double().permute(0, 2, 1, 3).reshape(-1, c["hkv"], d)
        flat[s["slots"]] = rows
        pools.append(flat.view(pool.shape[0], c["page"], c["hkv"], d).permute(0, 2, 1, 3).contiguous())
    return out[0].reshape(s["q"].shape), pools[0], pools[1]


def _exact_shared(s):
    """As if nothing were shared: every sequence by its own page list."""
    c = s["case"]
    hq, hkv, d, page = c["hq"], c["hkv"], c["dim"], c["page"]
    o = torch.zeros((s["total"], hq * d), dtype=torch.float64, device=DEV)
    lse = torch.zeros((s["total"], hq), dtype=torch.float64, device=DEV)
    cu, lens = s["cu_q"].tolist(), s["kv_len"].tolist()
    for b, n in enumerate(lens):
        lo, hi = cu[b], cu[b + 1]
        j = torch.arange(n, device=DEV)
        pages = s["table"][b, j // page].long()
        rank = torch.arange(hi - lo, device=DEV) if s["perm"] is None else s["perm"][lo:hi].long()
        for h in range(hkv):
            k, v = s["K"][pages, h, j % page].double(), s["V"][pages, h, j % page].double()
            if c["int8"]:
                k, v = k * s["k_scale"][h].double(), v * s["v_scale"][h].double()
            for head in range(h * (hq // hkv), (h + 1) * (hq // hkv)):
                sc = s["q"][lo:hi, head * d:(head + 1) * d].double() @ k.T * s["scale"]
                sc[:, n - (hi - lo):].masked_fill_(rank[None, :] > rank[:, None], -math.inf)
                l = torch.logsumexp(sc, -1)
                lse[lo:hi, head] = l
                o[lo:hi, head * d:(head + 1) * d] = torch.exp(sc - l[:, None]) @ v
    return o, lse


def _exact_sample(s):
    logp = torch.zeros(s["x"].shape[0], dtype=torch.float64, device=DEV)
    par = [s[n].tolist() for n in ("temperature", "top_k", "top_p", "min_p", "u")]
    for b, (t, k, p, mp, u) in enumerate(zip(*par)):
        if t == 0:
            continue                                                             # one token, certain
        z = s["x"][b].double() / t
        order = torch.argsort(-z, stable=True)
        order = order[z[order] > -math.inf]
        if k > 0:
            order = order[:k]
        prob = torch.softmax(z[order], 0)
        n = order.shape[0] if p >= 1 else int((torch.cumsum(prob, 0) - prob < p).sum())
        n = max(1, min(n, int((prob >= mp * prob[0]).sum())))
        kept = torch.sort(order[:n]).values
        lp = torch.log_softmax(z[kept], 0)
        at = int((torch.cumsum(torch.exp(lp), 0) <= u).sum())
        logp[b] = lp[min(at, n - 1)]
    return None, logp, None


def exact(case, seed):
    if case["op"] == "plan":
        return None                                                              # whole numbers throughout
    s = prepare(case, seed)
    return {"rotary": _exact_rotary, "shared": _exact_shared, "sample": _exact_sample}[case["op"]](s)
