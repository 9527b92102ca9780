"""Plain 64-bit forms of the per-head norms with rotation and their gradients,
and the error bounds their tests use.  Test infrastructure only; shares nothing
with the kernels.

Bounds.  u is the unit roundoff of fp32 (2^-24), r half a step of the element
type relative to the value (bf16 2^-8, fp32 2^-24).

The inverse size 1 / sqrt(mean x^2 + eps): a sum of D squares, 16 one after the
other in a lane and at most 3 exchanges, each square and each sum one rounding:
20 u of the sum, whose terms are all positive; the sum with eps, the root and
the quotient one each; the root halves what came before: 10 u + 3 u < 14 u.  With
the product by gamma and by x a normed element is off by 16 u of itself.

Rotation: as in draft_ref: 7 u (|x| + |y|) of a pair, and 2 pi 3 2^-53 of the
turns for the angle.  Normed and rotated: (16 + 7) u (|x| + |y|); elements that
do not turn 16 u |x|.

Gradients.  g, dy turned back: eg = 7 u (|dy_x| + |dy_y|) and the angle's part.
n = r x is off by 15 u.  h = gamma g: |gamma| eg + u |h|.  m = mean(h n), a sum
of D products as above: mean(|n| |gamma| eg) + (20 + 15 + 3) u mean |h n|.
dx = r (h - n m): r (|gamma| eg + u |h| + |n| (error of m) + (15 + 1) u |n m|),
then r itself (14 u), its product and the difference: 16 u r (|h| + |n m|).
dgamma = sum of g n: |n| eg + (15 + 1) u |g n| a term, and N u of the sum of N
absolute terms.
"""
import numpy as np

U = 2.0 ** -24


def turned(x, pos, inv_freq, axis, pairs, sign=1.0):
    """x [S, H, D] at positions pos [axes, S]; returns (turned, |x| + |y| of each
    element's pair (|x| where it stays), bound on the angle's error)."""
    x = x.copy()
    size, err, stays = np.abs(x), np.zeros_like(x), np.ones(x.shape[-1], dtype=bool)
    half = len(inv_freq)
    for j in range(half):
        a, b = (2 * j, 2 * j + 1) if pairs else (j, j + half)
        ang = pos[axis[j]].astype(np.float64)[:, None] * float(inv_freq[j])
        c, s = np.cos(ang), sign * np.sin(ang)
        u, w = x[..., a].copy(), x[..., b].copy()
        x[..., a], x[..., b] = u * c - w * s, u * s + w * c
        size[..., a] = size[..., b] = np.abs(u) + np.abs(w)
        err[..., a] = err[..., b] = 3 * 2.0 ** -53 * np.abs(ang)
        stays[a] = stays[b] = False
    return x, size, err, stays


def forward(x, gamma, eps, rot, half):
    """y of x [S, H, D] (gamma None: 1, eps None: no norm; rot: (pos, inv_freq,
    axis, pairs) or None) and the bound on its error, half the output's
    half step."""
    n = x
    if eps is not None:
        n = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * (1.0 if gamma is None else gamma)
    own = 16 * U if eps is not None else 0.0
    if rot is None:
        y, bound = n, own * np.abs(n)
    else:
        y, size, err, stays = turned(n, *rot)
        bound = (own + np.where(stays, 0.0, 7 * U) + err) * size
    moved = (own > 0) | (bound > 0)
    return y, np.where(moved, bound + half * (np.abs(y) + bound), 0.0) * (1 + 1e-6)


def backward(x, dy, gamma, eps, rot, half):
    """dx, its bound, dgamma, its bound, of rows x, dy [S, H, D]."""
    D = x.shape[-1]
    if rot is None:
        g, eg = dy, np.zeros_like(dy)
    else:
        g, size, err, stays = turned(dy, *rot, sign=-1.0)
        eg = (np.where(stays, 0.0, 7 * U) + err) * size
    if eps is None:
        return g, np.where(eg > 0, eg + half * (np.abs(g) + eg), 0.0) * (1 + 1e-6), None, None
    gm = np.ones(D) if gamma is None else gamma
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n, h = r * x, gm * g
    m = (h * n).mean(-1, keepdims=True)
    em = (np.abs(n) * np.abs(gm) * eg).mean(-1, keepdims=True) + 38 * U * np.abs(h * n).mean(-1, keepdims=True)
    dx = r * (h - n * m)
    bound = r * (np.abs(gm) * eg + U * np.abs(h) + np.abs(n) * em + 16 * U * np.abs(n * m)) + \
        16 * U * r * (np.abs(h) + np.abs(n * m))
    bound += half * (np.abs(dx) + bound)
    N = x.shape[0] * x.shape[1]
    t = g * n
    dgamma = t.sum((0, 1))
    bg = (np.abs(n) * eg + 16 * U * np.abs(t)).sum((0, 1)) + N * U * np.abs(t).sum((0, 1))
    return dx, bound * (1 + 1e-6), dgamma, bg * (1 + 1e-6)
