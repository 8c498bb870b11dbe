"""Tree attention with more than 32 rows of tokens and query heads to a kv head, whose wavefronts share tiles of keys and values: the same
checks as with few rows, at the edges of these tiles, and scores so large that their powers of two would be infinite."""
import numpy as np
import pytest
import torch

import paper_2205_10034_amd as M
from attention_util import Paged, queries
from drafts_util import attend_tree, check_tree, firsts, tree_words
from oracle import drafts_oracle as O
from test_gpu_attention_tree import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [8, 64, 72, 128, 136, 256])
@pytest.mark.parametrize("n,G", [(9, 4), (16, 4), (17, 4), (33, 4), (64, 3), (3, 33), (64, 64)])
def test_rows_and_dimensions(n, G, D):
    lens = [n, n + 1, 31 + n, 300, 64, 65, 129]
    counts = [n, max(1, n - 1), n, n, max(1, n // 2), 1, n]
    run([max(a, b) for a, b in zip(lens, counts)], counts, G, 1, D, 16, "bf16")


@pytest.mark.parametrize("page,layout", [(1, "token_major"), (7, "head_major"), (32, "token_major"), (100, "head_major")])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_pages(D, page, layout):
    run([70, 1, 333, 64, 1100], [20, 1, 13, 5, 20], 8, 2, D, page, "bf16", layout)
    run([70, 1, 333, 64, 1100], [20, 1, 13, 5, 20], 8, 2, D, page, "bf16", layout, chain=True, pad=8)


@pytest.mark.parametrize("lens,counts", [([4000], [16]), ([9001], [40]), ([1, 5000, 3, 257], [1, 18, 3, 12]), ([700] * 20 + [0], [16] * 20 + [0]), ([300] + [20] * 99, [12] * 100)])
@pytest.mark.parametrize("D", [64, 128, 192])
def test_split_over_the_length(lens, counts, D):
    run(lens, counts, 8, 2, D, 64, "bf16")


@pytest.mark.parametrize("window,sinks", [(1, 0), (2, 4), (16, 0), (50, 33), (129, 4), (3, 100000), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_windows_and_sinks(D, window, sinks):
    run([16, 70, 129, 700, 5], [16, 9, 20, 12, 5], 8, 2, D, 16, "bf16", window=window, sinks=sinks)
    run([16, 70, 129, 700, 5], [16, 9, 20, 12, 5], 8, 2, D, 10, "bf16", "head_major", chain=True, window=window, sinks=sinks)


def test_cap_distance_and_scale():
    slopes = np.array([0.5, 0.0, 0.03, 3.0, -0.01, 1e-4, 0.25, 0.125], dtype=np.float32)
    lens, counts = [300, 41, 16, 77], [20, 16, 16, 3]
    for D in (64, 128, 256):
        run(lens, counts, 8, 2, D, 16, "bf16", softcap=5.0, gain=8.0)
        run(lens, counts, 8, 2, D, 16, "bf16", slopes=slopes)
        run(lens, counts, 8, 2, D, 16, "bf16", slopes=slopes, softcap=30.0, window=50, sinks=3, scale=0.3)
        run(lens, counts, 8, 2, D, 16, "bf16", gain=300.0)
        for scale in (-0.2, 0.0, 1e-30, 3e38):
            run([40, 20], [12, 16], 8, 2, D, 16, "bf16", scale=scale, gain=1e-36 if scale > 1 else 2.0)


def test_words_pages_and_lengths():
    rng = np.random.default_rng(3)
    counts = [15, 19, 64, 33]
    words = rng.integers(-2 ** 63, 2 ** 63, sum(counts), dtype=np.int64)
    words[::4] = 0
    for lens in ([50, 29, 100, 200], [15, 19, 64, 33]):
        run(lens, counts, 4, 2, 64, 16, "bf16", words=words)
        run(lens, counts, 4, 2, 128, 16, "bf16", words=words, window=7, sinks=2)
    p = Paged([100, 64, 300], 2, 128, 16, "bf16")
    table = p.table.copy()
    table[0, 2], table[1, :], table[2, 0], table[2, 7:12], table[2, 18] = -1, -5, p.n_pages, 2 ** 31 - 1, -2 ** 31
    run([100, 64, 300], [15, 13, 27], 8, 2, 128, 16, "bf16", table=table)
    run([48, 32, 16, 16], [14, 25, 16, 13], 8, 2, 64, 16, "bf16", spare_width=0, call_lens=[48, 1000, 3, -7])
    run([30, 40], [13, 14], 8, 2, 64, 16, "bf16", spare_rows=5, max_new=20)


@pytest.mark.parametrize("G", [3, 8])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_scores_whose_powers_are_beyond_float32(D, G):
    """Scores of 2.55e38 are finite, 1.44 times as much is not.  Only the largest count: the mean of their values."""
    lens, n = [200, 1000], 16
    p = Paged(lens, 1, D, 16, "bf16")
    big = float(np.sqrt(2.55e38 / D))
    q = torch.zeros(2 * n, G, D, dtype=torch.bfloat16)
    q[:] = big
    at = lambda s, j: (p.table[s, j // 16], j % 16, 0)  # noqa: E731
    for s, length in enumerate(lens):
        for j in range(length):
            p.k[at(s, j)] = 0.0
    best = {0: [7, 90, 150], 1: [3, 511, 900]}
    top = torch.tensor(big).bfloat16().float().item()
    assert D * top * top < float(np.finfo(np.float32).max) < D * top * top * 1.4427
    for s, js in best.items():
        for j in js:
            p.k[at(s, j)] = top
    out, _ = attend_tree(p.cache(), q, firsts([n, n]), lens, n, scale=1.0)
    for s, js in best.items():
        want = np.mean([p.v[at(s, j)] for j in js], axis=0)
        # equal weights of 1/3: a sum of three, and one rounding
        assert np.abs(out[s * n:(s + 1) * n] - want).max() <= 2.0 ** -8 * np.abs(want).max() + 2.0 ** -16 * 3 * np.abs(p.v).max(initial=0, where=~np.isnan(p.v))
    # all of them equal and as far below zero: the mean of all that a token sees
    for s, length in enumerate(lens):
        for j in range(length):
            p.k[at(s, j)] = -top
    out, lse = attend_tree(p.cache(), q, firsts([n, n]), lens, n, scale=1.0)
    check = O.tree(np.zeros_like(p.k), p.v, p.table, np.zeros((2 * n, G, D)), firsts([n, n]), lens, n, None, 1.0)
    assert np.abs(out - check[0]).max() <= 2.0 ** -8 * np.abs(check[0]).max() + 2.0 ** -16
    assert np.isfinite(lse).all() and (lse < -2.5e38).all()


@pytest.mark.parametrize("n,G", [(12, 4), (40, 3)])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_infinities_and_nan_in_unseen_drafts(D, n, G):
    """A branch's values that are not finite reach no other branch; keys of -infinity are not seen."""
    length = 100
    p = Paged([length], 2, D, 16, "bf16")
    place = lambda j: (p.table[0, j // 16], j % 16)  # noqa: E731
    words = np.array([1 << i for i in range(n)], dtype=np.int64)       # every token a branch of its own
    base = length - n
    p.v[place(base + 3)], p.v[place(base + 5)] = np.nan, np.inf
    p.k[place(base + 7)] = np.nan
    p.k[place(11)] = -np.inf
    q = queries(n, 2 * G, D, "bf16").abs()
    out, lse = attend_tree(p.cache(), q, [0, n], [length], n, words)
    clean_v, clean_k = np.nan_to_num(p.v, nan=0.0, posinf=0.0), np.nan_to_num(p.k, nan=0.0, neginf=-1e30)
    ref = O.tree(clean_k, clean_v, p.table, q.float().numpy(), [0, n], [length], n, words, D ** -0.5)
    rest = [i for i in range(n) if i not in (3, 5, 7)]
    assert np.isnan(out[3]).all() and not np.isfinite(out[5]).any() and np.isnan(out[7]).all() and np.isnan(lse[7]).all()
    assert np.abs(out[rest] - ref[0][rest]).max() < 2.0 ** -7 * np.abs(ref[0][rest]).max()


def test_results_do_not_change_streams_and_graphs():
    lens, counts = [1500, 17, 640], [17, 12, 20]
    p = Paged(lens, 2, 128, 16, "bf16")
    q, first, words = queries(49, 8, 128, "bf16"), firsts(counts), tree_words(counts)
    cache, qd = p.cache(), q.cuda()
    eager = attend_tree(cache, q, first, lens, 20, words)
    for _ in range(3):
        again = attend_tree(cache, q, first, lens, 20, words)
        assert np.array_equal(eager[0], again[0]) and np.array_equal(eager[1], again[1])
    dev = [torch.from_numpy(x).cuda() for x in (first, np.array(lens, dtype=np.int32), words)]
    ws = torch.empty(M.moe_attention_tree_workspace_bytes(cache, 8, 20), dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(qd), torch.empty(49, 8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    M.moe_attention_tree(cache, qd, dev[0], dev[1], out, ws, 20, visible=dev[2], lse=lse, stream=s)
    s.synchronize()
    assert np.array_equal(eager[0], out.float().cpu().numpy())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        M.moe_attention_tree(cache, qd, dev[0], dev[1], out, ws, 20, visible=dev[2], lse=lse)
    for now, counts in ((lens, [17, 12, 20]), ([1499, 3, 600], [1, 2, 18]), ([19, 17, 0], [14, 0, 2]), (lens, [17, 12, 20])):
        first, words = firsts(counts), np.zeros(49, dtype=np.int64)
        words[:sum(counts)] = tree_words(counts, seed=sum(now))
        for d, h in zip(dev, (first, np.array(now, dtype=np.int32), words)):
            d.copy_(torch.from_numpy(h))
        out.fill_(float("nan"))
        lse.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        eager = attend_tree(cache, q, first, now, 20, words)
        got = out.float().cpu().numpy()
        assert np.array_equal(eager[0], got, equal_nan=True) and np.array_equal(eager[1], lse.cpu().numpy(), equal_nan=True)
        check_tree(p, q, first, now, 20, got, lse.cpu().numpy(), words)


def test_places_beyond_32_bits():
    n_pages, page, hkv, D = 10000, 64, 16, 128       # 2.6e9 elements, 5.2 GB, in each pool
    far = [19998, 6, 16400, 18002]
    p = Paged([200], hkv, D, page, "bf16", spare_pages=0, spare_width=0)
    k = torch.full((2 * n_pages, page, hkv, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    v = torch.full((2 * n_pages, page, hkv, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    for i, f in enumerate(far):
        k[f] = torch.from_numpy(p.k[p.table[0, i]]).cuda()
        v[f] = torch.from_numpy(p.v[p.table[0, i]]).cuda()
    cache = M.KVCache(k, v, torch.tensor([far], dtype=torch.int32, device="cuda"))
    q, words = queries(20, 2 * hkv, D, "bf16"), tree_words([20])
    out, lse = attend_tree(cache, q, [0, 20], [200], 20, words)
    check_tree(p, q, [0, 20], [200], 20, out, lse, words)


@pytest.mark.parametrize("width,n_pages", [(0, 0), (0, 3), (2, 0)])
@pytest.mark.parametrize("n", [4, 20])
def test_caches_without_columns_or_pages(n, width, n_pages):
    """Nothing is there: outputs are zero, pages are not to be had, and nothing is read."""
    S, hkv, hq, D = 3, 2, 8, 64
    k = torch.zeros(n_pages, 16, hkv, D, dtype=torch.bfloat16, device="cuda")
    cache = M.KVCache(k, torch.zeros_like(k), torch.full((S, width), -1, dtype=torch.int32, device="cuda"))
    q = queries(S * n, hq, D, "bf16")
    out, lse = attend_tree(cache, q, firsts([n] * S), [50, 0, 7], n)
    assert not out.any() and np.isneginf(lse).all()
    refs, lens = torch.zeros(n_pages, dtype=torch.int32, device="cuda"), torch.tensor([40, 16, -1], dtype=torch.int32, device="cuda")
    ws, missing = torch.empty(M.moe_kv_pages_workspace_bytes(cache), dtype=torch.uint8, device="cuda"), torch.full((1,), -3, dtype=torch.int32, device="cuda")
    M.moe_kv_reserve(cache, refs, lens, ws, missing=missing)
    assert missing.item() == (3 if width else 0) and (cache.page_table == -1).all()
    one = lambda x: torch.tensor([x], dtype=torch.int32, device="cuda")  # noqa: E731
    M.moe_kv_fork(cache, refs, one(0), one(2), lens, ws, missing=missing)
    M.moe_kv_release(cache, refs, lens)
    M.moe_kv_compact(cache, lens, torch.zeros(S, 2, dtype=torch.int32, device="cuda"))
    assert lens.tolist() == [40, 16, 40] and missing.item() == 0 and not refs.any()
