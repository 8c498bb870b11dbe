"""Tree attention of scores far from zero: equal ones, single largest ones, and rows that differ by many orders."""
import numpy as np
import pytest
import torch

from attention_util import DT, HALF_STEP, Paged, queries
from drafts_util import attend_tree, check_tree, firsts
from oracle import drafts_oracle as O

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
FAR = [1e6, 1e9, 4e9, 1e12, 1e20, 1e30]


def at(p, s, j):
    return p.table[s, j // p.page], j % p.page, 0


def check_equal_or_gone(p, q, first, lens, n, out, lse, lse_bits=8.0):
    """Scores are exact numbers of float32, equal or so far apart that only the largest count: weights are the same number or 0.  Off are the
    sums of n terms, bfloat16 weights of two numbers, and one rounding; lse by some roundings of the score."""
    ref, ref_lse, mean_abs, *_ = O.tree(p.k, p.v, p.table, q.float().numpy(), first, lens, n, None, 1.0)
    assert np.isfinite(out).all() and np.isfinite(lse).all(), f"{(~np.isfinite(out)).sum()} outputs, {(~np.isfinite(lse)).sum()} lse of {lse.size} are not finite"
    size = (max(lens) + 16) * E
    tol = (size + (2.0 ** -17 if p.dtype == "bf16" else 0.0)) * mean_abs + HALF_STEP[p.dtype] * 1.01 * np.abs(ref)
    assert (np.abs(out - ref) <= tol).all(), f"out off by {np.abs(out - ref).max()}"
    assert (np.abs(lse - ref_lse) <= lse_bits * E * np.abs(ref_lse) + size).all(), f"lse off by {np.abs(lse - ref_lse).max()}"


@pytest.mark.parametrize("dtype,D,n,G", [("bf16", 64, 16, 3), ("bf16", 128, 16, 3), ("bf16", 256, 16, 3), ("bf16", 64, 32, 4), ("bf16", 128, 32, 4), ("bf16", 256, 32, 4), ("bf16", 128, 4, 4),
                                         ("f32", 64, 16, 4)])
@pytest.mark.parametrize("far", FAR + [-s for s in FAR])
def test_equal_and_single_largest_scores(far, dtype, D, n, G):
    lens = [n, 200, 1000]
    p = Paged(lens, 1, D, 16, dtype)
    q = torch.zeros(3 * n, G, D, dtype=DT[dtype])
    q[:, :, 0] = 1.0
    score = torch.tensor(far).to(DT[dtype]).item()
    for best in (None, {0: [0], 1: [77], 2: [2, 500]}):
        for s, length in enumerate(lens):
            for j in range(length):
                p.k[at(p, s, j)] = 0.0
                p.k[at(p, s, j)][0] = score if best is None or (j in best[s]) == (far > 0) else 0.0
        out, lse = attend_tree(p.cache(), q, firsts([n] * 3), lens, n, scale=1.0)
        check_equal_or_gone(p, q, firsts([n] * 3), lens, n, out, lse)


@pytest.mark.parametrize("rise", [8.0, 1e5, 3e9])
@pytest.mark.parametrize("D,n,G", [(64, 16, 3), (128, 16, 3), (256, 16, 3), (64, 32, 4), (128, 32, 4)])
def test_rows_whose_scores_are_far_beside_others(D, n, G, rise):
    """One head's scores grow by tiles from `rise` on to beyond 2^100, the others' stay as they usually are: these keep their accuracy whatever
    their neighbours in a wavefront do."""
    lens = [150, 1000]
    p = Paged(lens, 1, D, 16, "bf16")
    for s, length in enumerate(lens):
        for j in range(length):
            p.k[at(p, s, j)][0] = torch.tensor(rise * 4.0 ** min(j // 16, 40)).bfloat16().item()
    q = queries(2 * n, G, D, "bf16")
    q[:, :, 0] = 0.0
    q[:, 0] = 0.0
    q[:, 0, 0] = 1.0
    out, lse = attend_tree(p.cache(), q, firsts([n, n]), lens, n, scale=1.0)
    check_tree(p, q[:, 1:], firsts([n, n]), lens, n, out[:, 1:], lse[:, 1:], scale=1.0)
    check_equal_or_gone(p, q[:, :1], firsts([n, n]), lens, n, out[:, :1], lse[:, :1])
