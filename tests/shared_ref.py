"""Plain 64-bit forms of shared prefixes, entry weights and eviction, and the
error bounds their tests use.  Test infrastructure only; shares nothing with the
kernels.

Bounds (u = 2^-24).  Attention as derived in draft_ref, with the partial results
of one row counted among the sums: a logit is off by (D + 4) u scale sum |q k|, a
relative error e of every weight moves an output by 2 e sum p |v|, sums over N
keys in `parts` partial results add (N + 64 + parts) u, weights of bf16 calls
are rounded once, and so is the output.

Log-sum-exp: the largest error of a logit, the sum's (N + 64 + parts) u and its
exponentials' 2 u, and 4 u of |lse| + 20 for the logarithm, the maximum's product
with ln 2 and their sum (both are at most |lse| plus the logarithm of 2^28 keys).

Entry weights: exp(z - l) is off by the error of its exponent: (D + 4) u scale sum
|q k| of the logit, 3 u (|z| + |l|) of the two scalings to powers of 2 and their
difference, 2 u of the exponential.  N rows add N u of their sum, the former
weight one rounding more.
"""
import numpy as np

from draft_ref import U, slot_row


def entries(k_pages, v_pages, table, b, n):
    """(slots that have a page, their K and V [m, Hkv, D])."""
    where = [(c, slot_row(table, b, c, k_pages.shape[2], k_pages.shape[0])) for c in range(n)]
    where = [(c, w) for c, w in where if w]
    if not where:
        empty = np.zeros((0,) + k_pages.shape[1:2] + k_pages.shape[3:])
        return [], empty, empty
    pg, rw = np.array([w for _, w in where]).T
    return [c for c, _ in where], k_pages[pg, :, rw], v_pages[pg, :, rw]


def attention(q, sources, scale, half, parts):
    """One row q [Hq, D] over K, V [n, Hkv, D] of several sources: out, its
    bound, lse, its bound."""
    K, V = (np.concatenate([s[i] for s in sources]) for i in (0, 1))
    Hq, D = q.shape
    G = Hq // K.shape[1]
    out, bound = np.zeros((Hq, D)), np.zeros((Hq, D))
    lse, lse_bound = np.full(Hq, -np.inf), np.zeros(Hq)
    n = len(K)
    if n == 0:
        return out, bound, lse, lse_bound
    for h in range(Hq):
        k, v = K[:, h // G], V[:, h // G]
        z = scale * (k @ q[h])
        top = z.max()
        p = np.exp(z - top)
        lse[h] = top + np.log(p.sum())
        p /= p.sum()
        out[h] = p @ v
        logit = (D + 4) * U * scale * (np.abs(k) @ np.abs(q[h])).max()
        sums = (n + 64 + parts) * U
        weights = half if half > U else 0.0  # fp32 weights are not rounded again
        bound[h] = half * np.abs(out[h]) + (2 * (logit + 2 * U) + sums + weights) * (p @ np.abs(v))
        lse_bound[h] = logit + sums + 2 * U + 4 * U * (abs(lse[h]) + 20)
    return out, bound * (1 + 1e-6), lse, lse_bound * (1 + 1e-6)


def gathered(q, lse, seen, K, scale, had):
    """Weights of entries K [n, D] of one KV head from rows q [rows, D] with lse
    [rows], of which row i sees the first seen[i] entries (seen of entries that
    have a page), added to had [n]; returns (weights, bound)."""
    D = q.shape[1]
    z = scale * (q @ K.T)
    size = scale * (np.abs(q) @ np.abs(K).T)
    use = (np.arange(K.shape[0])[None] < seen[:, None]) & ~np.isneginf(lse)[:, None]
    l = np.where(np.isneginf(lse), 0.0, lse)[:, None]
    p = np.where(use, np.exp(np.where(use, z - l, 0.0)), 0.0)
    off = (D + 4) * U * size + 3 * U * (np.abs(z) + np.abs(l)) + 2 * U
    total = had + p.sum(0)
    return total, ((p * off).sum(0) + len(q) * U * p.sum(0) + U * np.abs(total)) * (1 + 1e-6)


def kept_slots(w, keep, first, recent):
    """Slots that stay of a row of weights w [L]."""
    L = len(w)
    n = min(L, keep)
    f = min(first, n)
    r = min(recent, n - f)
    if n == L:
        return list(range(L))
    mid = sorted(range(f, L - r), key=lambda c: (0 if w[c] == w[c] else 1, -w[c] if w[c] == w[c] else 0.0, c))
    return list(range(f)) + sorted(mid[:n - f - r]) + list(range(L - r, L))
