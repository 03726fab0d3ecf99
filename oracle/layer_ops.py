"""fp64 NumPy definitions of what runs between a layer's projections.

Inputs are NumPy arrays (fp16 values, int32 ids); every result is fp64,
unrounded.  Nothing here shares code with the HIP path.
"""

from __future__ import annotations

import numpy as np


def rope_table(inv_freq, positions: int, scale: float = 1.0) -> np.ndarray:
    """[positions x rot / 2 x 2]: (cos, sin)(p w_i) * scale."""
    angle = np.arange(positions, dtype=np.float64)[:, None] * np.asarray(inv_freq, dtype=np.float64)
    return np.stack([np.cos(angle), np.sin(angle)], axis=2) * scale


def rms_norm(x, weight, eps: float) -> np.ndarray:
    x = np.asarray(x, dtype=np.float64)
    return x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64)


def rope(x, table, positions, interleaved: bool, norm=None, eps: float = 1e-6) -> np.ndarray:
    """x [T x H x D], each head normed (if ``norm``) and its pairs turned; a
    position outside the table gives NaN."""
    y = np.asarray(x, dtype=np.float64).copy()
    if norm is not None:
        y = rms_norm(y, norm, eps)
    if table is None:
        return y
    half = table.shape[1]
    for t, p in enumerate(positions):
        if not 0 <= p < table.shape[0]:
            y[t] = np.nan
            continue
        for i in range(half):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
            c, s = float(table[p, i, 0]), float(table[p, i, 1])
            u, v = y[t, :, a].copy(), y[t, :, b].copy()
            y[t, :, a], y[t, :, b] = u * c - v * s, v * c + u * s
    return y


def append(cache, rows, slots) -> np.ndarray:
    """The cache [pages x page_size x H x D] with ``rows`` [T x H x D] at ``slots``."""
    out = np.asarray(cache, dtype=np.float64).copy()
    pages, size = out.shape[:2]
    for t, s in enumerate(slots):
        if 0 <= s < pages * size:
            out[s // size, s % size] = rows[t]
    return out


def paged_attention(q, k_cache, v_cache, pages, q_start, kv_len, scale: float, causal: bool = True, window: int = 0):
    """(out [T x Hq x D], lse [T x Hq], mass [T x Hq x D]): ``mass`` is the
    softmax-weighted sum of |v|, the scale of the rounding errors of the
    weights.  Only the keys a token sees are touched.  Tokens of no request
    are NaN."""
    T, Hq, D = q.shape
    size, Hkv = k_cache.shape[1], k_cache.shape[2]
    out, mass = np.full((T, Hq, D), np.nan), np.full((T, Hq, D), np.nan)
    lse = np.full((T, Hq), np.nan)
    for b in range(len(kv_len)):
        n, kv = int(q_start[b + 1] - q_start[b]), int(kv_len[b])
        j = np.arange(kv)
        page = pages[b][j // size]
        keys = k_cache[page, j % size].astype(np.float64)
        values = v_cache[page, j % size].astype(np.float64)
        for i in range(n):
            t, pos = int(q_start[b]) + i, kv - n + i
            end = min(pos + 1, kv) if causal else kv
            begin = max(0, pos - window + 1) if window else 0
            for h in range(Hq):
                if begin >= end:
                    out[t, h], lse[t, h], mass[t, h] = 0.0, -np.inf, 0.0
                    continue
                g = h // (Hq // Hkv)
                s = scale * (keys[begin:end, g] @ q[t, h].astype(np.float64))
                m = s.max()
                e = np.exp(s - m)
                p = e / e.sum()
                lse[t, h] = m + np.log(e.sum())
                out[t, h] = p @ values[begin:end, g]
                mass[t, h] = p @ np.abs(values[begin:end, g])
    return out, lse, mass


def residual_norm(x, y=None, weight=None, eps: float = 1e-5, post_weight=None, gate=None, scale: float = 1.0):
    """(x_new, h); h is None without ``weight``."""
    x = np.asarray(x, dtype=np.float64)
    if y is not None:
        u = np.asarray(y, dtype=np.float64)
        if post_weight is not None:
            u = rms_norm(u, post_weight, eps)
        if gate is not None:
            u = u * np.asarray(gate, dtype=np.float64)
        x = x + scale * u
    return x, (None if weight is None else rms_norm(x, weight, eps))


def lora(x, adapters, A, B, scales, base=None):
    """(y, mass): y = base + s B (A x); ``mass`` = |s| |B| (|A| |x|), the scale of
    the summation's rounding errors."""
    M, N = x.shape[0], B.shape[1]
    y = np.zeros((M, N)) if base is None else np.asarray(base, dtype=np.float64).copy()
    mass = np.zeros((M, N))
    for m, a in enumerate(adapters):
        if 0 <= a < A.shape[0]:
            xm, Aa, Ba = (np.asarray(t, dtype=np.float64) for t in (x[m], A[a], B[a]))
            y[m] += float(scales[a]) * (Ba @ (Aa @ xm))
            mass[m] = abs(float(scales[a])) * (np.abs(Ba) @ (np.abs(Aa) @ np.abs(xm)))
    return y, mass
