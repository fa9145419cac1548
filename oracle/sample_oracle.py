"""Sampling from its definition, in float64 NumPy, one row at a time.  Shares no code with the GPU path."""
import numpy as np


def sample(x, temperature, u, top_k=0, top_p=1.0, min_p=0.0, most=float(np.finfo(np.float32).max)):
    """(token, log probability, kept indices ascending) of one row x [V]; token -1 where nothing can be kept.

    Parameters are the float32 / int32 values of the call; most: the largest finite number of x's type, which +infinity counts as.
    """
    x = np.where(np.isnan(x), -np.inf, np.minimum(np.asarray(x, np.float64), most)) + 0.0
    t, p, mp, u = (float(np.float32(v)) for v in (temperature, top_p, min_p, u))
    order = np.argsort(-x, kind="stable")
    order = order[x[order] > -np.inf]
    if order.size == 0:
        return -1, -np.inf, order
    if not t > 0:
        return int(order[0]), 0.0, order[:1]
    top = x[order[0]]
    gap = np.where(x[order] == top, 0.0, x[order] - top)
    w = np.where(gap == 0.0, 1.0, np.where(np.isinf(gap), 0.0, np.exp(gap / t)))
    n = order.size if not 0 < top_k < x.size else min(top_k, order.size)
    order, w = order[:n], w[:n]
    if p < 1:
        before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
        n = min(n, int((before < p * w.sum()).sum()))
    if mp > 0 and not np.isinf(t):      # (every weight is 1 there, and min_p at most 1)
        n = min(n, int((gap[:n] >= t * np.log(min(mp, 1.0))).sum()))
    n = max(n, 1)
    kept = np.sort(order[:n])
    wk = np.zeros(x.size)
    wk[order[:n]] = w[:n]
    run = np.cumsum(wk[kept])
    u = min(max(u, 0.0), float(np.float32(0.99999994)))
    j = int((run <= u * run[-1]).sum())
    return int(kept[j]), float(np.log(wk[kept[j]] / run[-1])), kept
