"""Plain 64-bit forms of the steps of several new tokens, and the error bounds
their tests use.  Test infrastructure only; shares nothing with the kernels.

Bounds.  u is the unit roundoff of fp32 (2^-24), r half a step of the element
type relative to the value (bf16 2^-8, fp32 2^-24).

Rotation: x cos a - y sin a with cos and sin off by at most 4 u (the fp32 angle
in half turns is off by u / 2, times pi; the functions by 2 u), two products and
a sum of relative error u each: at most 7 u (|x| + |y|), then one rounding of
the result.  In the reduction to turns the product of the position and the
frequency is off by three 64-bit roundings of its t turns: 2 pi 3 2^-53 |t|.

Attention: a logit is a sum of D products in fp32, off by at most (D + 4) u
scale sum |q k| (its scaling and the reference maximum included); a relative
error e of every weight moves an output by at most 2 e sum p |v|.  Sums over N
keys in fp32 (with the rescaling of the running sums and the merge of splits)
add (N + 64) u sum p |v|, rounding the weights to the element type r sum p |v|,
the exponential 2 u, and the output one rounding.
"""
import numpy as np
import torch

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def f64(t):
    return t.detach().to("cpu", torch.float64).numpy()


def rotate(x, pos, inv_freq, pairs):
    """x [..., H, D] at positions pos [...]; returns (rotated, |x| + |y| of each
    element's pair, bound on the angle's error)."""
    x = x.copy()
    size = np.abs(x)
    err = np.zeros_like(x)
    half = len(inv_freq)
    for j in range(half):
        a, b = (2 * j, 2 * j + 1) if pairs else (j, j + half)
        ang = pos.astype(np.float64)[..., None] * float(inv_freq[j])
        c, s = np.cos(ang), np.sin(ang)
        u, w = x[..., a].copy(), x[..., b].copy()
        x[..., a], x[..., b] = u * c - w * s, u * s + w * c
        size[..., a] = size[..., b] = np.abs(u) + np.abs(w)
        err[..., a] = err[..., b] = 3 * 2.0 ** -53 * np.abs(ang)
    return x, size, err


def slot_row(table, b, slot, page_size, num_pages):
    """(page, row) of a cache slot, or None where the table has no page for it."""
    i = slot // page_size
    if i >= table.shape[1]:
        return None
    page = int(table[b, i])
    return (page, slot % page_size) if 0 <= page < num_pages else None


def tree(q, k_pages, v_pages, table, lens, nodes, see, scale, half):
    """q [B, n, Hq, D]; see(b, i, j): node i of sequence b sees node j.
    Returns (out, bound) as float64 arrays; rows past nodes[b] are NaN."""
    B, n, Hq, D = q.shape
    P, Hkv, ps, _ = k_pages.shape
    out = np.full(q.shape, np.nan)
    bound = np.zeros(q.shape)
    for b in range(B):
        if nodes[b] == 0:
            continue
        slots = [slot_row(table, b, c, ps, P) for c in range(lens[b] + nodes[b])]
        where = [c for c, w in enumerate(slots) if w]  # slots that have a page
        if not where:
            out[b, :nodes[b]] = 0.0
            continue
        pg, rw = np.array([slots[c] for c in where]).T
        hide = np.array([[c >= lens[b] and not see(b, i, c - lens[b]) for c in where] for i in range(nodes[b])])
        keys = np.sum(~hide, axis=1)[:, None]
        for h in range(Hq):
            K, V = k_pages[pg, h * Hkv // Hq, rw], v_pages[pg, h * Hkv // Hq, rw]
            x = q[b, :nodes[b], h]
            z = np.where(hide, -np.inf, scale * (x @ K.T))
            top = z.max(1, keepdims=True)
            p = np.exp(z - np.where(np.isinf(top), 0.0, top))
            p /= np.where(keys, p.sum(1, keepdims=True), 1.0)
            out[b, :nodes[b], h] = p @ V
            a = p @ np.abs(V)
            size = np.where(hide, 0.0, np.abs(x) @ np.abs(K).T).max(1, keepdims=True)
            e = (D + 4) * U * scale * size + 2 * U
            weights = half if half > U else 0.0  # fp32 weights are not rounded again
            bound[b, :nodes[b], h] = half * np.abs(out[b, :nodes[b], h]) + (2 * e + (keys + 64) * U + weights) * a
    return out, bound * (1 + 1e-6)


def ancestors(parents):
    see = []
    for i, p in enumerate(parents):
        see.append({i} | (see[p] if p >= 0 else set()))
    return see
