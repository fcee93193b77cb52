"""Plain float64 definitions of the 8-bit unit caches and the paged memory:
the e4m3 format with power-of-two scales, the append (norm of each head,
rotation) and the attention over a memory.  Test infrastructure only."""
from __future__ import annotations

import numpy as np


def _code_values() -> np.ndarray:
    """Value of every e4m3 code byte (0x7f and 0xff: NaN)."""
    b = np.arange(256)
    e, m = (b >> 3) & 15, (b & 7).astype(np.float64)
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v[(b & 127) == 127] = np.nan
    return np.where(b >= 128, -v, v)


CODES = _code_values()
_POSITIVE = CODES[:127]                       # ascending


def scale_bytes(x: np.ndarray) -> np.ndarray:
    """Scale byte of every group (last axis) of x: the least k >= -126 with amax <= 448 * 2^k, plus 127."""
    x = np.asarray(x, np.float64)
    bad = ~np.isfinite(x).all(-1)
    amax = np.where(bad, 0.0, np.abs(np.where(np.isfinite(x), x, 0.0)).max(-1))
    k = np.full(amax.shape, -126)
    for step in (128, 64, 32, 16, 8, 4, 2, 1):          # the largest k that is still too small, plus one
        more = amax > 448.0 * 2.0 ** (k + step - 1.0)
        k = np.where(more, k + step, k)
    return np.where(bad, 255, k + 127).astype(np.uint8)


def quantise(x: np.ndarray):
    """(code bytes of x's shape, scale bytes) of groups along the last axis; nearest code, ties to the even byte."""
    x = np.asarray(x, np.float64)
    s = scale_bytes(x)
    v = np.abs(np.where(s[..., None] == 255, 0.0, x)) * 2.0 ** (127.0 - s[..., None])
    hi = np.clip(np.searchsorted(_POSITIVE, v), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = _POSITIVE[hi] - v, v - _POSITIVE[lo]
    c = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    c = np.where(_POSITIVE[hi] == v, hi, c).astype(np.uint8)
    c = np.where(np.signbit(x), c | 128, c)
    return np.where(s[..., None] == 255, 127, c).astype(np.uint8), s


def dequantise(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return CODES[codes] * s[..., None]


def cache_write(r, x, refresh, codes, scales):
    """In place on codes [N][H][E] and scales [N][H][E/32]; returns y (float64)."""
    on = np.ones(len(r), bool) if refresh is None else np.asarray(refresh) != 0
    c, s = quantise(r.reshape(*scales.shape, 32))
    codes[on], scales[on] = c.reshape(codes.shape)[on], s[on]
    return np.where(on[:, None, None], x.astype(np.float64) + r, x)


def cache_add(codes, scales, x, reuse):
    y = np.asarray(x, np.float64).copy()
    for u in range(len(codes)):
        on = np.ones(len(y), bool) if reuse is None else np.asarray(reuse[u]) != 0
        y[on] += dequantise(codes[u].reshape(*scales[u].shape, 32), scales[u]).reshape(y.shape)[on]
    return y


def normed_and_turned(x, gain, eps, pos, base):
    """x [rows][heads][D] with its RMS norm (gain None: none) and rotation (base None: none)."""
    x = np.asarray(x, np.float64)
    D = x.shape[-1]
    if gain is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(gain, np.float64)
    if base is None:
        return x
    w = float(base) ** (-2.0 * np.arange(D // 2) / D)
    ang = np.asarray(pos, np.float64)[:, None, None] * w
    a, b = x[..., :D // 2], x[..., D // 2:]
    return np.concatenate([a * np.cos(ang) - b * np.sin(ang), b * np.cos(ang) + a * np.sin(ang)], -1)


def attend(q, k, v, n_kv, scale, causal, window):
    """One sequence: q [m][Hq][D], k and v [len][Hk][D].  Returns out, the mean of |v| under the
    same weights (what the rounding of a weight can move) and the largest sum of |q||k| * scale."""
    m, Hq, D = q.shape
    n = len(k)
    out, size, dots = np.zeros((m, Hq, D)), np.zeros((m, Hq, D)), 0.0
    key = np.arange(n)
    for j in range(m):
        hi = min(n, n - m + j + 1) if causal else n
        lo = max(0, hi - window) if window else 0
        see = key[lo:max(hi, lo)]
        if hi <= lo:
            continue
        for h in range(Hq):
            g = h * n_kv // Hq
            s = k[see, g] @ q[j, h] * scale
            with np.errstate(invalid="ignore"):
                p = np.exp(s - s.max())
                p /= p.sum()
                out[j, h], size[j, h] = p @ v[see, g], p @ np.abs(v[see, g])
            dots = max(dots, float(np.nan_to_num((np.abs(k[see, g]) @ np.abs(q[j, h])).max())) * abs(scale))
    return out, size, dots
