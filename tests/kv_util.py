"""Paged caches for the tests: random sequences scattered over shuffled pages, with what must not be read made poisonous."""
import numpy as np
import torch

from paper_2502_00425_b200 import binding as B

DEV = "cuda"


class Paged:
    """Sequences of `lens` keys in a paged cache.  Slots behind a sequence's end hold NaN (bf16) or extreme codes (int8), table
    entries behind its last page hold page numbers outside the cache, one page belongs to nobody.
    k[b], v[b]: float64 [len, heads, dim], the values the cache stands for."""

    def __init__(self, lens, n_kv, dim, page, int8=False, layout="head", seed=0, extra_pages=2, device=DEV):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.page, self.int8, self.n_kv, self.dim = list(lens), page, int8, n_kv, dim
        need = [-(-n // page) for n in lens]
        n_pages = sum(need) + 1
        order = torch.randperm(n_pages, generator=g).tolist()
        width = max(need + [1]) + extra_pages
        table = torch.full((len(lens), width), n_pages + 7, dtype=torch.int32)
        table[:, -1] = -5
        if int8:
            pools = [torch.full((n_pages, n_kv, page, dim), 127, dtype=torch.int8) for _ in range(2)]
            self.k_scale, self.v_scale = ((torch.rand(n_kv, generator=g) * 0.5 + 0.5) / 40 for _ in range(2))
        else:
            pools = [torch.full((n_pages, n_kv, page, dim), float("nan"), dtype=torch.bfloat16) for _ in range(2)]
            self.k_scale = self.v_scale = None
        self.k, self.v = [], []
        at = 0
        for b, n in enumerate(lens):
            pages = order[at:at + need[b]]
            at += need[b]
            table[b, :need[b]] = torch.tensor(pages, dtype=torch.int32)
            for pool, out, scale in zip(pools, (self.k, self.v), (self.k_scale, self.v_scale)):
                x = torch.randn((n, n_kv, dim), generator=g)
                rows = (x * 40).round().clamp(-128, 127).to(torch.int8) if int8 else x.to(torch.bfloat16)
                for i, pg in enumerate(pages):
                    part = rows[i * page:(i + 1) * page]
                    pool[pg, :, :part.shape[0]] = part.transpose(0, 1)
                val = rows.double()
                out.append((val * scale.double()[:, None] if int8 else val).numpy())
        if layout == "token":     # [page, slot, head, dim] in memory
            pools = [p.permute(0, 2, 1, 3).contiguous().to(device).permute(0, 2, 1, 3) for p in pools]
        elif layout == "padded":  # rows, heads and pages further apart than they need to be
            wide = [torch.zeros((n_pages, n_kv + 1, page + 3, dim + 16), dtype=p.dtype, device=device) for p in pools]
            for w, p in zip(wide, pools):
                w[:, :n_kv, :page, :dim] = p.to(device)
            pools = [w[:, :n_kv, :page, :dim] for w in wide]
        else:
            pools = [p.to(device) for p in pools]
        self.K, self.V = pools
        self.table = table.to(device)
        self.kv_len = torch.tensor(lens, dtype=torch.int32, device=device)
        s = (lambda t: None if t is None else t.to(device))
        self.cache = B.KVCache(self.K, self.V, s(self.k_scale), s(self.v_scale))

    def rows(self, pool, b, n=None):
        """The first n cached rows of sequence b as the pool holds them: [n, heads, dim] on the host."""
        n = self.lens[b] if n is None else n
        pool, table = pool.cpu(), self.table.cpu()
        j = torch.arange(n)
        return pool[table[b, j // self.page].long(), :, j % self.page]


def cu(new, device=DEV):
    return torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device=device)


def aifs_perm(rng, new):
    """perm of ragged chunks, each reordered as AIFS reorders a random mix of visual and text tokens."""
    out = []
    for n in new:
        vis = rng.random(n) < 0.6
        out.append(np.concatenate([np.flatnonzero(vis), np.flatnonzero(~vis)]))
    return out
