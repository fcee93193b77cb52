"""Plain float64 definitions of the latent memory: append (norm of the latent, rotation of
the key part and the queries' parts), attention of absorbed queries over latents, and the
expansion of latents to a head's keys and values.  Test infrastructure only."""
from __future__ import annotations

import numpy as np


def normed(c, gain, eps):
    """c [rows][rank] over its root mean square, times gain (None: c as it is)."""
    c = np.asarray(c, np.float64)
    return c if gain is None else c / np.sqrt((c * c).mean(-1, keepdims=True) + eps) * np.asarray(gain, np.float64)


def turned(x, pos, base):
    """x [rows][...][64], the pairs (i, i + 32) turned by pos [rows] times base^(-i / 32) (base None: not)."""
    x = np.asarray(x, np.float64)
    if base is None:
        return x
    half = x.shape[-1] // 2
    ang = np.asarray(pos, np.float64)[:, None] * float(base) ** (-np.arange(half) / half)
    ang = ang.reshape(ang.shape[:1] + (1,) * (x.ndim - 2) + ang.shape[1:])
    z = (x[..., :half] + 1j * x[..., half:]) * np.exp(1j * ang)
    return np.concatenate([z.real, z.imag], -1)


def attend(q, x, rank, scale, causal, window):
    """One sequence: q [m][H][rank + 64] over x [len][rank + 64].  Returns out [m][H][rank], the mean of |c| under the
    same weights (what the rounding of a weight can move) and the largest sum of |q||x| * scale."""
    m, H, n = len(q), q.shape[1], len(x)
    out, size, dots = np.zeros((m, H, rank)), np.zeros((m, H, rank)), 0.0
    for j in range(m):
        hi = min(n, n - m + j + 1) if causal else n
        lo = max(0, hi - window) if window else 0
        if hi <= lo:
            continue
        see = x[lo:hi]
        with np.errstate(invalid="ignore"):
            s = q[j] @ see.T * scale
            p = np.exp(s - s.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            out[j], size[j] = p @ see[:, :rank], p @ np.abs(see[:, :rank])
            dots = max(dots, float(np.nan_to_num(np.abs(q[j]) @ np.abs(see).T).max()) * abs(scale))
    return out, size, dots


def expand(x, w_k, w_v):
    """Keys [len][H][64 + 64] and values [len][H][128] of x [len][rank + 64]."""
    rank = w_k.shape[-1]
    c, k = x[:, :rank], x[:, rank:]
    keys = np.einsum("tr,hdr->thd", c, w_k)
    return np.concatenate([keys, np.repeat(k[:, None], len(w_k), 1)], -1), np.einsum("tr,hdr->thd", c, w_v)
