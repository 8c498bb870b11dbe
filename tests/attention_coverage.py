"""Which places the decode attention took, read off its outputs: with scores that are all equal, lse is the logarithm of how many
there were, and values that are 1 in one dimension for each block of 16 places and 0 elsewhere make out the share of each dimension's
blocks.  A tile that is lost, counted twice or taken for another shows in one of the two, whatever the length."""
import numpy as np
import torch

import paper_2205_10034_amd as M
from attention_util import DT, HALF_STEP

BLOCK = 16


def kept_places(n, window, missing_pages, page):
    j = np.arange(max(0, n - window) if window else 0, n)
    return j[~np.isin(j // page, missing_pages)]


def counts(places, D):
    """How many of these places mark each dimension."""
    return np.bincount(places // BLOCK % D, minlength=D).astype(np.float64)


def accepted(out, lse, taken, D, dtype):
    """Whether out [heads, D] and lse [heads] of a sequence are those of `taken` (dimension -> places).  Weights are powers of two and
    counts below 2^24 exact in float32; what rounds is the reciprocal of the sum, the product with it, and the type: 2 * 2^-24 and half a
    step.  lse: a logarithm to 2 units and two roundings, of a number below 32: 8 * 2^-24 of itself."""
    n = taken.sum()
    if n == 0:
        return bool((out == 0).all() and np.isneginf(lse).all())
    want, want_lse = taken / n, np.log(n)
    tol = want * (2 * 2.0 ** -24 + (HALF_STEP[dtype] if dtype == "bf16" else 0.0)) * 1.01
    return bool((np.abs(out - want) <= tol).all() and (np.abs(lse - want_lse) <= 8 * 2.0 ** -24 * want_lse + 2.0 ** -24).all())


class Marked:
    """Sequences of the given lengths whose values mark their places, over a pool of at least `pool_mb` megabytes; all else is NaN."""

    def __init__(self, lens, hkv, D, page, dtype, layout="token_major", pool_mb=0, missing=(), spare_width=1, seed=0):
        g = torch.Generator().manual_seed(seed)
        es = 2 if dtype == "bf16" else 4
        per_seq = [-(-n // page) for n in lens]
        n_pages = max(sum(per_seq) + 2, int(pool_mb * 1e6 / (2 * page * hkv * D * es)) + 1)
        order = torch.randperm(n_pages, generator=g).to(torch.int32)
        table = torch.full((len(lens), max(per_seq + [0]) + spare_width), -1, dtype=torch.int32)
        first = 0
        for s, n in enumerate(per_seq):
            table[s, :n] = order[first:first + n]
            first += n
        places = [torch.arange(n) for n in lens]
        at = torch.cat([table[s].long()[j // page] * page + j % page for s, j in enumerate(places)]).cuda()
        mark = torch.cat([j // BLOCK % D for j in places]).cuda()
        for s, column in missing:
            table[s, column] = -1 if column % 2 else n_pages
        k = torch.full((n_pages * page, hkv, D), float("nan"), dtype=DT[dtype], device="cuda")
        v = k.clone()
        k[at], v[at] = 1.0, 0.0
        v[at, :, mark] = 1.0
        k, v = (t.view(n_pages, page, hkv, D) for t in (k, v))
        if layout == "head_major":
            k, v = (t.transpose(1, 2).contiguous() for t in (k, v))
        self.cache = M.KVCache(k, v, table.cuda(), layout=layout)
        self.lens, self.page, self.D, self.dtype, self.missing = lens, page, D, dtype, missing

    def check(self, hq, window=0):
        S = len(self.lens)
        q = torch.randn(S, hq, self.D, generator=torch.Generator().manual_seed(1)).to(DT[self.dtype]).cuda()
        out, lse = torch.full_like(q, float("nan")), torch.full((S, hq), float("nan"), device="cuda")
        ws = torch.full((M.moe_attention_decode_workspace_bytes(self.cache, hq),), 255, dtype=torch.uint8, device="cuda")
        M.moe_attention_decode(self.cache, q, torch.tensor(self.lens, dtype=torch.int32, device="cuda"), out, ws, scale=0.0, window=window, lse=lse)
        out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
        for s, n in enumerate(self.lens):
            taken = counts(kept_places(n, window, [c for b, c in self.missing if b == s], self.page), self.D)
            assert accepted(out[s], lse[s], taken, self.D, self.dtype), f"sequence {s} of {n} places: lse {lse[s][:4]}, expected {np.log(max(taken.sum(), 1e-300))}"
