"""Independent float64 NumPy statement of a step of drafted tokens: attention for a tree of them over a paged cache, the
places of the accepted ones, pages by counts, and the log-probabilities of tokens with their gradient.  Test
infrastructure only: the product package never imports it."""
from __future__ import annotations

import numpy as np

from .attention_oracle import place


def cut(token_first, seq_lens, T, max_new, capacity):
    """(first row, new tokens, base, places) of every sequence."""
    out = []
    for s in range(len(seq_lens)):
        first = min(max(int(token_first[s]), 0), T)
        n = min(max(min(int(token_first[s + 1]), T) - first, 0), max_new)
        places = min(max(int(seq_lens[s]), 0), capacity)
        out.append((first, n, max(0, places - n), places))
    return out


def words_of(n, words):
    """What each of n tokens sees of the others, as sets."""
    return [set(range(i + 1)) if words is None else {j for j in range(n) if int(words[i]) >> j & 1} for i in range(n)]


def tree(k, v, table, q, token_first, seq_lens, max_new, visible=None, scale=1.0, softcap=0.0, window=0, sinks=0, slopes=None):
    """k, v [pages, page_size, kv heads, D]; q [T, H, D].  out and lse (NaN: a row of no sequence), and what bounds of rounding
    need, as in attention_oracle.decode; the number of places seen by each token."""
    T, H, D = q.shape
    n_pages, page_size, hkv, _ = k.shape
    G = H // hkv
    out, mean_abs = np.full((T, H, D), np.nan), np.zeros((T, H, D))
    lse, dot_abs, z_abs, seen = np.full((T, H), np.nan), np.zeros((T, H)), np.zeros((T, H)), np.zeros(T)
    for s, (first, n, base, places) in enumerate(cut(token_first, seq_lens, T, max_new, table.shape[1] * page_size)):
        see = words_of(n, None if visible is None else [int(w) & (2 ** 64 - 1) for w in visible[first:first + n]])
        pos = [base + len(see[i] - {i}) for i in range(n)]
        where = [place(table, n_pages, page_size, s, j) for j in range(places)]
        for i in range(n):
            at = []
            for j in range(places):
                if where[j] is None or (j >= base and j - base not in see[i]):
                    continue
                away = pos[i] - (j if j < base else pos[j - base])
                if not window or away < window or j < sinks:
                    at.append((j, away))
            t = first + i
            out[t], lse[t], seen[t] = 0.0, -np.inf, len(at)
            if not at:
                continue
            pages, rows = np.array([where[j][0] for j, _ in at]), np.array([where[j][1] for j, _ in at])
            away = np.array([a for _, a in at], dtype=np.float64)
            for h in range(H):
                kk, vv = np.float64(k[pages, rows, h // G]), np.float64(v[pages, rows, h // G])
                with np.errstate(invalid="ignore"):
                    z = scale * (kk @ np.float64(q[t, h]))
                    if softcap:
                        z = softcap * np.tanh(z / softcap)
                    if slopes is not None:
                        z = z - float(slopes[h]) * away
                top = z.max()
                if top == -np.inf:
                    continue
                w = np.exp(z - top)
                lse[t, h] = top + np.log(w.sum())
                w /= w.sum()
                out[t, h], mean_abs[t, h] = w @ vv, w @ np.abs(vv)
                dot_abs[t, h] = abs(scale) * (np.abs(kk) @ np.abs(np.float64(q[t, h]))).max()
                z_abs[t, h] = np.abs(z[np.isfinite(z)]).max(initial=0.0) + (0 if slopes is None else abs(float(slopes[h])) * np.abs(away).max())
    return out, lse, mean_abs, dot_abs, z_abs, seen


def compact(pools, table, base, keep):
    """New pools [pages, page_size, kv heads, D] and lengths."""
    new, lens = [p.copy() for p in pools], []
    n_pages, page_size = pools[0].shape[:2]
    for s in range(len(base)):
        n = 0
        while n < len(keep[s]) and keep[s][n] >= 0:
            a = place(table, n_pages, page_size, s, int(base[s]) + int(keep[s][n]))
            b = place(table, n_pages, page_size, s, int(base[s]) + n)
            if a is not None and b is not None:
                for p, q in zip(pools, new):
                    q[b] = p[a]
            n += 1
        lens.append(int(base[s]) + n)
    return new, lens


class Pages:
    """A page table and its counts on the host."""

    def __init__(self, table, refs, page_size):
        self.table, self.refs, self.P = [list(map(int, r)) for r in table], list(map(int, refs)), page_size

    def valid(self, entry):
        return 0 <= entry < len(self.refs)

    def take(self):
        for p, r in enumerate(self.refs):
            if r == 0:
                self.refs[p] = 1
                return p
        return -1

    def drop(self, s, places):
        for c in range(-(-max(places, 0) // self.P), len(self.table[s])):
            if self.valid(self.table[s][c]):
                self.refs[self.table[s][c]] -= 1
            self.table[s][c] = -1

    def release(self, lens):
        for s, n in enumerate(lens):
            self.drop(s, int(n))

    def fork(self, src, dst, lens):
        """Copies to make, (page, page, places), and how many pages were not to be had; lens follows."""
        S, copies, missing = len(self.table), [], 0
        pairs = [(int(a), int(b)) for a, b in zip(src, dst) if 0 <= a < S and 0 <= b < S and a != b]
        sources, taken = {a for a, _ in pairs}, set()
        pairs = [(a, b) for a, b in pairs if b not in sources and not (b in taken or taken.add(b))]
        size = lambda s: min(max(int(lens[s]), 0), len(self.table[s]) * self.P)  # noqa: E731
        for a, b in pairs:
            self.drop(b, 0)
        for a, b in pairs:
            for c in range(size(a) // self.P):
                self.table[b][c] = self.table[a][c]
                if self.valid(self.table[b][c]):
                    self.refs[self.table[b][c]] += 1
        for a, b in pairs:
            whole, begun = divmod(size(a), self.P)
            if begun and self.valid(self.table[a][whole]):
                self.table[b][whole] = page = self.take()
                missing += page < 0
                if page >= 0:
                    copies.append((self.table[a][whole], page, begun))
            lens[b] = lens[a]
        return copies, missing

    def reserve(self, lens, more):
        missing = 0
        for s, n in enumerate(lens):
            for c in range(min(-(-(int(n) + more) // self.P), len(self.table[s])) if n >= 0 else 0):
                if not self.valid(self.table[s][c]):
                    self.table[s][c] = self.take()
                    missing += self.table[s][c] < 0
        return missing

    def consistent(self):
        """Counts are what the table says."""
        named = [0] * len(self.refs)
        for row in self.table:
            for e in row:
                if self.valid(e):
                    named[e] += 1
        return named == self.refs


def logprobs(x, ids, scale=1.0, K=0):
    """Of rows x [T, V]: logp, lse, entropy, top ids and their log-probabilities, probabilities."""
    T, V = x.shape
    z = np.asarray(x, dtype=np.float64) * float(np.float32(scale))
    with np.errstate(invalid="ignore", divide="ignore"):
        top = np.nanmax(np.where(np.isnan(z), -np.inf, z), axis=1, keepdims=True)
        bad = (np.isnan(z) | (z == np.inf)).any(1)
        d = np.where(np.isneginf(z), -np.inf, z - np.where(np.isneginf(top), 0.0, top))
        e = np.exp(d)
        s = e.sum(1, keepdims=True)
        lp = d - np.log(s)
        p = e / s
    lp[np.isneginf(top[:, 0])], p[np.isneginf(top[:, 0])] = -np.inf, 0.0
    lse = top[:, 0] + np.where(np.isneginf(top[:, 0]), 0.0, np.log(np.where(s > 0, s, 1.0))[:, 0])
    entropy = -np.where(p > 0, p * np.where(p > 0, lp, 0.0), 0.0).sum(1)
    lp[bad], lse[bad], entropy[bad], p[bad] = np.nan, np.nan, np.nan, np.nan
    logp = np.zeros(T)
    for t in range(T):
        if 0 <= ids[t] < V:
            logp[t] = lp[t, ids[t]]
    key = np.where(np.isnan(x), -np.inf, np.asarray(x, dtype=np.float64))
    order = np.stack([np.lexsort((np.arange(V), -key[t], np.isnan(x[t]))) for t in range(T)])[:, :K] if T else np.zeros((0, K), int)
    return logp, lse, entropy, order, np.take_along_axis(lp, order, 1), p


def logprobs_gradient(x, ids, scale=1.0, d_logp=None, d_entropy=None, d_lse=None):
    """d_x of sum d_logp logp + d_entropy entropy + d_lse lse, and how large its terms are."""
    T, V = x.shape
    zeros = np.zeros(T)
    _, lse, entropy, _, _, p = logprobs(x, ids, scale)
    scale = float(np.float32(scale))
    g = np.where((np.asarray(ids) >= 0) & (np.asarray(ids) < V), zeros if d_logp is None else np.asarray(d_logp, dtype=np.float64), 0.0)
    ge, gl = (zeros if d is None else np.asarray(d, dtype=np.float64) for d in (d_entropy, d_lse))
    with np.errstate(invalid="ignore", divide="ignore"):
        lp = np.where(p > 0, np.log(np.where(p > 0, p, 1.0)), 0.0)
        d = p * (gl - g)[:, None] - ge[:, None] * p * (lp + entropy[:, None])
        size = p * (np.abs(g) + np.abs(gl) + np.abs(ge) * (np.abs(entropy) + 1))[:, None] + np.abs(ge)[:, None] * p * np.abs(lp)
    for t in range(T):
        if np.isneginf(lse[t]) or (g[t] == 0 and ge[t] == 0 and gl[t] == 0):
            d[t] = size[t] = 0.0
        elif g[t] != 0:
            d[t, ids[t]] += g[t]
            size[t, ids[t]] += abs(g[t])
    return scale * d, scale * size
