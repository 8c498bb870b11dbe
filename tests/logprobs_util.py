"""Bounds of the log-probabilities and of their gradient, element by element, from what the arithmetic does: a weight's own error times how much
it moves a result, instead of the largest that any could have."""
import numpy as np

from attention_util import HALF_STEP
from oracle import drafts_oracle as O

E = 2.0 ** -24


class Rows:
    """Rows h [T, V] of finite logits in 64 bits, and how far a forward call may be off.

    A weight exp(z_j - m): difference, its product with c and c itself are each rounded, for references up to 6 behind the row's, and brought to
    others four times at most; a power is off by a unit: delta_j = E (8 (|d_j| + 6) + 8) of it.  A lane adds up n terms: its roundings, of
    either sign, have a standard deviation of E sqrt(n) / 3, and what 64 or more lanes have is joined in some ten steps more: E (sqrt(n) + 16)."""

    def __init__(self, h, ids, scale=1.0):
        V = h.shape[1]
        self.h, self.ids, self.scale = h, np.asarray(ids), float(np.float32(scale))
        z = np.asarray(h, dtype=np.float64) * self.scale
        self.top = z.max(1)
        self.d = z - self.top[:, None]
        w = np.exp(self.d)
        self.log_s = np.log(w.sum(1))
        self.lse = self.top + self.log_s
        self.lp = self.d - self.log_s[:, None]
        self.p = np.exp(self.lp)
        self.entropy = -(self.p * self.lp).sum(1)
        self.delta = E * (8 * (np.abs(self.d) + 6) + 8)
        self.sums = E * (np.sqrt(16 * np.ceil(V / 4096) + 48) + 16)
        self.log_sum_off = (self.p * self.delta).sum(1) + self.sums + 2 * E * self.log_s
        self.lse_off = self.log_sum_off + E * (np.abs(self.top) + np.abs(self.lse))
        a = (self.p * (np.abs(self.d) + 2)).sum(1)
        self.entropy_off = (self.p * self.delta * np.abs(self.lp + self.entropy[:, None])).sum(1) + self.sums * (1 + a) + E * (2 * self.log_s + 8 * a + self.entropy)

    def logp(self):
        t = np.arange(len(self.h))
        have = (self.ids >= 0) & (self.ids < self.h.shape[1])
        at = np.where(have, self.ids, 0)
        want, d = np.where(have, self.lp[t, at], 0.0), np.abs(self.d[t, at])
        return want, np.where(have, self.log_sum_off + E * (2 * d + np.abs(want)), 0.0)

    def check_forward(self, got):
        logp, logp_off = self.logp()
        for name, want, off in (("lse", self.lse, self.lse_off), ("logp", logp, logp_off), ("entropy", self.entropy, self.entropy_off)):
            bad = ~(np.abs(got[name] - want) <= off + 1e-37)
            assert not bad.any(), f"{name} off at {np.argwhere(bad)[:4].tolist()}: {got[name][bad][:4]} for {want[bad][:4]}, allowed {off[bad][:4]}"

    def check_gradient(self, got, dtype, d_logp=None, d_entropy=None, d_lse=None):
        """p = exp(x scale - lse), off by lse's error and its own power; of rows whose |lse| is above 1024 (float32: 64) by that of a new sum.  The
        token's own g (1 - p): off by that of p, or, where 1 - p is below (|lse| + 8) 2^-13 (float32: 2^-7), by that of the sum of all others."""
        h, ids, scale = self.h, self.ids, self.scale
        T, V = h.shape
        zeros = np.zeros(T)
        f = lambda x: zeros if x is None else np.asarray(x, dtype=np.float64)  # noqa: E731
        g, ge, gl = np.where((ids >= 0) & (ids < V), f(d_logp), 0.0), f(d_entropy), f(d_lse)
        narrow = dtype == "bf16"
        lse_off = np.where(np.abs(self.lse) > (1024 if narrow else 64), self.log_sum_off, self.lse_off)
        lp_off = lse_off[:, None] + E * (2 * np.abs(self.lp) + 2)
        p_off = lp_off + E * (2 + 2 * np.abs(self.lp))
        c = lambda x: np.abs(x)[:, None]  # noqa: E731
        H = self.entropy[:, None]
        want = self.p * (gl - g)[:, None] - ge[:, None] * self.p * (self.lp + H)
        off = self.p * (p_off * (c(g) + c(gl) + c(ge) * np.abs(self.lp + H)) + c(ge) * (lp_off + c(self.entropy_off)) + 4 * E * (c(g) + c(gl) + c(ge) * (np.abs(self.lp) + H)))
        for t in np.flatnonzero(g):
            i = ids[t]
            others = np.exp(self.d[t])
            others[i] = 0.0
            rest, p, lp = others.sum() / np.exp(self.log_s[t]), self.p[t, i], self.lp[t, i]
            lp = np.log1p(-rest) if rest < 0.5 else lp
            rest_off = rest * (((others * self.delta[t]).sum() / max(others.sum(), 1e-300)) + self.sums + 16 * E)
            by_rest = -lp < 0.98 * (abs(self.lse[t]) + 8) * (2.0 ** -13 if narrow else 2.0 ** -7)
            here = rest_off + 2 * E * abs(lp) if by_rest else lp_off[t, i]
            want[t, i] = g[t] * rest + p * (gl[t] - ge[t] * (lp + self.entropy[t]))
            off[t, i] = abs(g[t]) * (rest_off if by_rest else p * p_off[t, i] + 2 * E) + p * (
                (here + 8 * E) * (abs(gl[t]) + abs(ge[t]) * abs(lp + self.entropy[t])) + abs(ge[t]) * (here + self.entropy_off[t] + 2 * E * (abs(lp) + self.entropy[t])))
        none = (g == 0) & (ge == 0) & (gl == 0)
        want[none], off[none] = 0.0, 0.0
        tol = scale * off * 1.01 + HALF_STEP[dtype] * 1.01 * np.abs(scale * want) + 1e-37
        bad = ~(np.abs(got - scale * want) <= tol)
        assert not bad.any(), f"{bad.sum()} off, at {np.argwhere(bad)[:4].tolist()}: {got[bad][:4]} for {(scale * want)[bad][:4]}, allowed {tol[bad][:4]}"


def confident(T, V, dtype, level, left, seed=0):
    """Rows of logits around `level` less some, in which token ids[t] has all but about `left` of the probability (as far as the type can say)."""
    import torch
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    rng = np.random.default_rng(seed + V)
    h = torch.from_numpy(np.float32(level - 12 + 2 * rng.standard_normal((T, V)))).to(dt).float().numpy()
    ids = rng.integers(0, V, T)
    if V > 1:
        for t in range(T):
            others = np.delete(np.float64(h[t]), ids[t])
            m = others.max()
            h[t, ids[t]] = torch.tensor(m + np.log(np.exp(others - m).sum()) - np.log(left)).to(dt).item()
    return h, ids
