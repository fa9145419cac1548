"""The key/value-cache operators from their definitions, in float64 NumPy, one sequence and head at a time.

Plain and slow, sharing no code with the GPU path.  Every function also returns what the tolerances of the tests are
made of: the sums of magnitudes that roundings are relative to.
"""
import numpy as np


def visible(n_new, n_all, perm=None):
    """bool [n_new, n_all]: row i of a chunk sees the context (the first n_all - n_new keys) and the chunk's rows that
    do not come after it: those with an index up to i, or with perm[j] <= perm[i] when the chunk stands in AIFS order."""
    rank = np.arange(n_new) if perm is None else np.asarray(perm, np.int64)
    ctx = n_all - n_new
    out = np.zeros((n_new, n_all), bool)
    for j in range(n_all):
        out[:, j] = True if j < ctx else rank[j - ctx] <= rank
    return out


def attention(q, k, v, scale, perm=None):
    """One head: q [n_new, D], k, v [n_all, D] -> (o, lse, p, abs_pv, score_mag).

    A row without keys: zeros and -inf.  Values of keys that a row does not see do not enter (not even as 0 * inf).
    abs_pv[i, d] = sum_j p |v|;  score_mag[i] = max over visible j of scale * sum_d |q| |k|.
    """
    q, k, v = (np.asarray(a, np.float64) for a in (q, k, v))
    n, m = q.shape[0], k.shape[0]
    see = visible(n, m, perm)
    o, lse = np.zeros((n, v.shape[1])), np.full(n, -np.inf)
    p, abs_pv, mag = np.zeros((n, m)), np.zeros((n, v.shape[1])), np.zeros(n)
    for i in range(n):
        idx = np.flatnonzero(see[i])
        if idx.size == 0:
            continue
        s = scale * (k[idx] @ q[i])
        top = s.max()
        e = np.exp(s - top)
        lse[i] = top + np.log(e.sum())
        p[i, idx] = e / e.sum()
        with np.errstate(invalid="ignore"):
            o[i] = p[i, idx] @ v[idx]
            abs_pv[i] = p[i, idx] @ np.abs(v[idx])
        mag[i] = scale * (np.abs(k[idx]) @ np.abs(q[i])).max()
    return o, lse, p, abs_pv, mag


def weights(q_heads, k, lse_heads, scale, perm=None):
    """Softmax weight of every key over all rows and the query heads of one key/value head: float64 [n_all]."""
    k = np.asarray(k, np.float64)
    w = np.zeros(k.shape[0])
    for q, lse in zip(q_heads, lse_heads):
        q = np.asarray(q, np.float64)
        see = visible(q.shape[0], k.shape[0], perm)
        for i in range(q.shape[0]):
            idx = np.flatnonzero(see[i])
            if idx.size:
                w[idx] += np.exp(scale * (k[idx] @ q[i]) - float(lse[i]))
    return w


def norm_rope(x, gain, eps, pos, base, half):
    """Heads x [T, H, D]: RMSNorm (gain None: skipped), then the rotary embedding.  Returns (y, mag): mag is the sum of the
    magnitudes of the two normed channels that a result is made of."""
    x = np.asarray(x, np.float64)
    T, H, D = x.shape
    if gain is not None:
        x = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps) * np.asarray(gain, np.float64)
    y, mag = np.empty_like(x), np.empty_like(x)
    for i in range(D // 2):
        a, b = (i, i + D // 2) if half else (2 * i, 2 * i + 1)
        ang = np.asarray(pos, np.float64) * base ** (-2.0 * i / D)
        c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., a] * s + x[..., b] * c
        mag[..., a] = mag[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return y, mag


def rope_theta(r, base, factor=1.0, original=0, fast=32.0, slow=1.0):
    """Radians per position of the r / 2 pairs; with an original context, pairs between `slow` and `fast` turns in it are scaled in
    proportion, those above stay."""
    out = []
    for i in range(r // 2):
        t = base ** (-2.0 * i / r)
        wavelength = 2 * np.pi / t
        keep = 0.0 if not original else np.clip((original / wavelength - slow) / (fast - slow), 0.0, 1.0)
        out.append(keep * t + (1 - keep) * t / factor)
    return np.array(out)


def norm_rope_scaled(x, gain, eps, pos, theta, half, amp):
    """norm_rope of the first 2 len(theta) channels with given frequencies, times amp; the others are normed only."""
    x = np.asarray(x, np.float64)
    if gain is not None:
        x = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps) * np.asarray(gain, np.float64)
    r = 2 * len(theta)
    y, mag = x.copy(), np.abs(x)
    for i, t in enumerate(theta):
        a, b = (i, i + r // 2) if half else (2 * i, 2 * i + 1)
        z = (x[..., a] + 1j * x[..., b]) * (amp * np.exp(1j * np.asarray(pos, np.float64) * t))[:, None]
        y[..., a], y[..., b] = z.real, z.imag
        mag[..., a] = mag[..., b] = abs(amp) * (np.abs(x[..., a]) + np.abs(x[..., b]))
    return y, mag


def keep(w, n, budget, n_first, n_last):
    """Indices (ascending) of the keys one head keeps of its n keys with weights w [n]."""
    if n <= budget:
        return np.arange(n)
    always = [j for j in range(n) if j < n_first or j >= n - n_last]
    rest = [j for j in range(n) if n_first <= j < n - n_last]
    key = lambda j: (1, 0.0, j) if np.isnan(w[j]) else (0, -float(w[j]), j)
    rest.sort(key=key)
    return np.array(sorted(always + rest[:budget - n_first - n_last]), np.int64)
