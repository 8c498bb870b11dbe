"""Independent float64 NumPy statement of the attention half of a decoded token: rotary positions, the paged cache and
the attention of one new token over it.  Test infrastructure only: the product package never imports it."""
from __future__ import annotations

import numpy as np


def rotary(x, positions, freqs, axis_pairs, interleaved=False, inverse=False):
    """x [T, H, D]; positions [axes, T]; freqs [pairs]; every pair as a complex number times exp(+-i angle)."""
    y = np.array(x, dtype=np.float64)
    half = len(freqs)
    axis = np.repeat(np.arange(len(axis_pairs)), axis_pairs)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        angle = np.asarray(positions, dtype=np.float64)[axis[i]] * float(freqs[i])
        z = (y[:, :, a] + 1j * y[:, :, b]) * np.exp((-1j if inverse else 1j) * angle)[:, None]
        y[:, :, a], y[:, :, b] = z.real, z.imag
    return y


def place(table, n_pages, page_size, s, p):
    """(page, row) of place p of sequence s, or None where there is none."""
    if not (0 <= s < table.shape[0] and 0 <= p and p // page_size < table.shape[1]):
        return None
    page = int(table[s, p // page_size])
    return (page, p % page_size) if 0 <= page < n_pages else None


def decode(k, v, table, q, lens, scale, softcap=0.0, window=0, slopes=None):
    """k, v [pages, page_size, kv heads, D]; q [S, H, D].  Returns out, lse and what bounds of rounding need: per (sequence,
    head) the weighted mean of |v|, the largest sum of |q k| and the largest |z|."""
    S, H, D = q.shape
    n_pages, page_size, hkv, _ = k.shape
    G = H // hkv
    out, mean_abs = np.zeros((S, H, D)), np.zeros((S, H, D))
    lse, dot_abs, z_abs = np.full((S, H), -np.inf), np.zeros((S, H)), np.zeros((S, H))
    for s in range(S):
        n = int(min(max(int(lens[s]), 0), table.shape[1] * page_size))
        at = [(j, place(table, n_pages, page_size, s, j)) for j in range(max(0, n - window) if window else 0, n)]
        at = [(j, w) for j, w in at if w is not None]
        if not at:
            continue
        pages, rows, js = np.array([w[0] for _, w in at]), np.array([w[1] for _, w in at]), np.array([j for j, _ in at])
        for h in range(H):
            kk, vv = np.float64(k[pages, rows, h // G]), np.float64(v[pages, rows, h // G])
            with np.errstate(invalid="ignore"):
                z = scale * (kk @ np.float64(q[s, h]))
                if softcap:
                    z = softcap * np.tanh(z / softcap)
                if slopes is not None:
                    z = z - float(slopes[h]) * (n - 1 - js)
            top = z.max()
            if top == -np.inf:
                continue
            w = np.exp(z - top)
            lse[s, h] = top + np.log(w.sum())
            w /= w.sum()
            out[s, h], mean_abs[s, h] = w @ vv, w @ np.abs(vv)
            dot_abs[s, h] = abs(scale) * (np.abs(kk) @ np.abs(np.float64(q[s, h]))).max()
            z_abs[s, h] = np.abs(z[np.isfinite(z)]).max(initial=0.0) + (0 if slopes is None else abs(float(slopes[h])) * n)
    return out, lse, mean_abs, dot_abs, z_abs
