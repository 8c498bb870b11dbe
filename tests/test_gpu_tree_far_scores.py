"""Tree attention of scores far from zero: equal ones, single largest ones, rows that differ by many orders, and large values under them."""
import numpy as np
import pytest
import torch

from attention_util import DT, HALF_STEP, Paged, queries
from drafts_util import attend_tree, check_tree, firsts, tree_words
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


@pytest.mark.parametrize("dtype,D,n,G,far", [("bf16", 64, 4, 2, 128), ("bf16", 128, 8, 4, 128), ("bf16", 256, 4, 2, 64), ("f32", 64, 4, 2, 64), ("f32", 256, 12, 3, 64),
                                             ("bf16", 64, 16, 4, 128), ("bf16", 128, 16, 3, 64), ("bf16", 256, 16, 4, 64), ("bf16", 64, 16, 8, 128), ("bf16", 128, 32, 4, 64)])
@pytest.mark.parametrize("base,more", [(0.0, 5.40625), (2.0 ** 17, 5.40625), (-2.0 ** 17, 5.40625), (2.0 ** 20, 5.375), (2.0 ** 24, 6.0), (2.0 ** 26, 8.0), (-2.0 ** 26, 8.0)])
def test_large_values_under_rising_scores(base, more, dtype, D, n, G, far):
    """Values near the type's largest whose keys are a little better than those of tiles before: no weight is above 1, so the mean of finite values
    is finite.  Scores and their differences are exact; weights are off by their power's 16 units at most, sums of n by n * 2^-24."""
    lens = [max(far + 1, n), 257, 900]
    p = Paged(lens, 1, D, 16, dtype)
    big = torch.tensor(3e38).to(DT[dtype]).item()
    for s, length in enumerate(lens):
        for j in range(length):
            p.k[at(p, s, j)], p.v[at(p, s, j)] = 0.0, 1.0
            p.k[at(p, s, j)][0] = base
        p.k[at(p, s, far)][1], p.v[at(p, s, far)] = more, big
        p.v[at(p, s, far)][1::2] = -big
    q = torch.zeros(3 * n, G, D, dtype=DT[dtype])
    q[:, :, :2] = 1.0
    words = tree_words([n] * 3)
    out, lse = attend_tree(p.cache(), q, firsts([n] * 3), lens, n, words, scale=1.0)
    ref, ref_lse, mean_abs, *_ = O.tree(p.k, p.v, p.table, q.float().numpy(), firsts([n] * 3), lens, n, words, 1.0)
    lost = int((~np.isfinite(out)).sum())
    assert lost == 0, f"{lost} of {out.size} are not finite"
    tol = (2 * (max(lens) + 64) * E + (2.0 ** -16 if dtype == "bf16" else 0.0)) * mean_abs + HALF_STEP[dtype] * 1.01 * np.abs(ref)
    # fast units: exponents are powers of two of numbers up to 2^18, whose difference c2 = scale log2(e) scales with one rounding
    tol += 2 * 16 * E * mean_abs
    assert (np.abs(out - ref) <= tol).all(), f"off by {(np.abs(out - ref) / tol).max()} times what is allowed"
    assert (np.abs(lse - ref_lse) <= 8 * E * np.abs(ref_lse) + (max(lens) + 64) * E).all()
