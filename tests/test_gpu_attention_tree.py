"""Attention of drafted tokens over a paged cache against the definition in 64 bits: trees and chains, uneven numbers of tokens, windows
and sinks, lengths around tiles and pages, head groups and dimensions of every kind, missing pages, NaN wherever nothing may be
read into a result."""
import numpy as np
import pytest
import torch

import paper_2205_10034_amd as M
from attention_util import DT, Paged, attend, queries
from drafts_util import attend_tree, check_tree, firsts, tree_words
from oracle import drafts_oracle as O

pytestmark = pytest.mark.gpu

RAGGED = [1, 2, 5, 15, 16, 17, 31, 33, 64, 127, 129, 300]
COUNTS = [1, 2, 3, 4, 1, 7, 2, 3, 9, 1, 5, 6]


def run(lens, counts, hq, hkv, D, page, dtype, layout="token_major", chain=False, words="tree", table=None, gain=2.0, pad=0, one_pool=False, spare_width=1, max_new=None,
        call_lens=None, spare_rows=0, **kw):
    print(lens[:8], counts[:8], hq, hkv, D, page, dtype, layout, chain, kw, flush=True)
    p = Paged(lens, hkv, D, page, dtype, layout, pad=pad, one_pool=one_pool, spare_width=spare_width)
    T = sum(counts) + spare_rows
    q = queries(T, hq, D, dtype, gain=gain)
    first = firsts(counts)
    visible = None
    if not chain:
        visible = np.zeros(T, dtype=np.int64)
        visible[:sum(counts)] = tree_words(counts) if isinstance(words, str) else words
    max_new = max_new or max(counts + [1])
    call_lens = lens if call_lens is None else call_lens
    out, lse = attend_tree(p.cache(table), q, first, call_lens, max_new, visible, **kw)
    check_tree(p, q, first, call_lens, max_new, out, lse, visible, table=table, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [1, 7, 16, 32, 100])
@pytest.mark.parametrize("layout", ["token_major", "head_major"])
def test_lengths_and_pages(page, layout, dtype):
    run(RAGGED, COUNTS, 4, 2, 64, page, dtype, layout)


@pytest.mark.parametrize("D,dtype", [(8, "bf16"), (24, "bf16"), (64, "bf16"), (72, "bf16"), (80, "bf16"), (96, "bf16"), (128, "bf16"), (136, "bf16"), (192, "bf16"),
                                     (256, "bf16"), (4, "f32"), (12, "f32"), (60, "f32"), (64, "f32"), (68, "f32"), (100, "f32"), (128, "f32"), (132, "f32"),
                                     (256, "f32")])
def test_head_dimensions(D, dtype):
    run([5, 70, 333], [5, 3, 8], 6, 2, D, 16, dtype)
    run([1, 200], [1, 20], 4, 2, D, 9, dtype, "head_major", softcap=20.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G", [1, 2, 5, 8, 15, 16, 17, 33])
@pytest.mark.parametrize("n", [1, 6, 64])
def test_head_groups_and_counts(n, G, dtype):
    run([70, 64, 150], [n, max(1, n - 3), max(1, n // 2)], 2 * G, 2, 32, 16, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,counts", [([1], [1]), ([4000], [3]), ([9001], [20]), ([1, 5000, 3, 257], [1, 8, 3, 2]), ([513] * 20, [2] * 20)])
def test_split_over_the_length(lens, counts, dtype):
    run(lens, counts, 8, 2, 64, 64, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_sequences(dtype):
    rng = np.random.default_rng(5)
    counts = rng.integers(0, 5, 400).tolist()
    run([int(n + rng.integers(0, 60)) for n in counts], counts, 2, 1, 64, 16, dtype)
    run([700] + [9] * 99, [3] * 100, 4, 4, 64, 16, dtype, spare_width=100)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 4), (16, 0), (50, 33), (129, 4), (100000, 7), (3, 100000), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_windows_and_sinks(window, sinks, dtype):
    run(RAGGED + [700], COUNTS + [12], 4, 2, 64, 16, dtype, window=window, sinks=sinks)
    run(RAGGED + [700], COUNTS + [12], 4, 2, 64, 10, dtype, "head_major", chain=True, window=window, sinks=sinks)


def test_sinks_without_a_window_change_nothing():
    run(RAGGED, COUNTS, 4, 2, 64, 16, "bf16", sinks=5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_words_that_are_no_trees(dtype):
    rng = np.random.default_rng(3)
    counts = [5, 9, 64, 3, 33]
    words = rng.integers(-2 ** 63, 2 ** 63, sum(counts), dtype=np.int64)
    words[::4] = 0                       # sees the cache only; a sequence without one: nothing
    for lens in ([50, 9, 100, 3, 200], [5, 9, 64, 3, 33]):
        run(lens, counts, 4, 2, 64, 16, dtype, words=words)
        run(lens, counts, 4, 2, 64, 16, dtype, words=words, window=7, sinks=2, slopes=np.array([0.1, 0.5, -0.2, 0.0], dtype=np.float32))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cap_and_distance_bias(dtype):
    slopes = np.array([0.5, 0.0, 0.03, 3.0, -0.01, 1e-4, 0.25, 0.125], dtype=np.float32)
    run(RAGGED, COUNTS, 8, 4, 64, 16, dtype, softcap=5.0, gain=8.0)
    run(RAGGED, COUNTS, 8, 4, 64, 16, dtype, slopes=slopes)
    run(RAGGED, COUNTS, 8, 4, 64, 16, dtype, slopes=slopes, softcap=30.0, window=50, sinks=3, scale=0.3)
    run([5000], [11], 8, 1, 64, 16, dtype, slopes=slopes)
    run([40], [4], 8, 4, 64, 16, dtype, scale=-0.2)
    run([40, 1], [4, 1], 8, 4, 64, 16, dtype, scale=0.0)
    run([70, 9], [4, 2], 8, 4, 64, 16, dtype, softcap=1e-38)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores(dtype):
    run([1, 40, 700], [1, 9, 3], 4, 2, 64, 16, dtype, gain=300.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_missing_pages(dtype):
    lens, counts = [100, 64, 300, 40, 20], [5, 3, 7, 10, 20]
    p = Paged(lens, 2, 64, 16, dtype)
    table = p.table.copy()
    table[0, 2] = -1                       # in the middle
    table[1, :] = -5                       # all of them: nothing is seen
    table[2, 0] = p.n_pages                # one past the pool
    table[2, 7:12] = 2 ** 31 - 1
    table[3, 2] = -2 ** 31                 # the last one, of new tokens
    table[4, 0] = -1                       # all that the first new tokens see
    run(lens, counts, 4, 2, 64, 16, dtype, table=table)
    run(lens, counts, 4, 2, 64, 16, dtype, table=table, window=20, sinks=3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lengths_outside_the_table_and_below_the_counts(dtype):
    lens = [48, 32, 16, 16]
    # clamped to the table's 48 places (of which one page is not there), to zero, and shorter than their new tokens
    run(lens, [4, 5, 6, 3], 4, 2, 64, 16, dtype, spare_width=0, call_lens=[48, 1000, 3, -7])
    run(lens, [4, 5, 6, 3], 4, 2, 64, 16, dtype, spare_width=0, call_lens=[0, 2 ** 31 - 1, 6, -2 ** 31], window=4, sinks=1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_no_sequence_and_bad_offsets(dtype):
    run([30, 40], [3, 4], 4, 2, 64, 16, dtype, spare_rows=5)
    run([30, 40], [3, 9], 4, 2, 64, 16, dtype, max_new=4)                   # tokens beyond max_new belong to nobody
    p = Paged([30, 40, 20], 2, 64, 16, dtype)
    q = queries(10, 4, 64, dtype)
    for first in ([0, 3, 2, 6], [-5, 4, 8, 100], [12, 12, 12, 12], [9, 2 ** 31 - 1, -2 ** 31, 4], [0, 0, 0, 0]):
        out, lse = attend_tree(p.cache(), q, first, p.lens, 8)
        # rows that two sequences claim hold the result of either: nothing more is said of them
        claims = np.zeros(10, dtype=int)
        for row, n, _, _ in O.cut(first, p.lens, 10, 8, p.table.shape[1] * 16):
            claims[row:row + n] += 1
        ref = O.tree(p.k, p.v, p.table, q.float().numpy(), first, p.lens, 8, None, 0.125)
        out[claims > 1], lse[claims > 1] = ref[0][claims > 1], ref[1][claims > 1]
        check_tree(p, q, first, p.lens, 8, out, lse)


def test_strides():
    run(RAGGED, COUNTS, 4, 2, 64, 16, "bf16", pad=8)
    run(RAGGED, COUNTS, 4, 2, 64, 16, "bf16", "head_major", pad=24, one_pool=True)
    run(RAGGED, COUNTS, 4, 2, 64, 7, "f32", one_pool=True, pad=4)
    p = Paged([5, 40, 130], 2, 64, 16, "bf16")
    counts = [2, 3, 4]
    q, first = queries(9, 4, 64, "bf16"), firsts(counts)
    wide = torch.full((9, 9, 72), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 2:6, :64] = q.cuda()
    outs = torch.full((9, 6, 80), 7.0, dtype=torch.bfloat16, device="cuda")
    cache = p.cache()
    ws = torch.empty(M.moe_attention_tree_workspace_bytes(cache, 4, 4), dtype=torch.uint8, device="cuda")
    lse = torch.empty(9, 4, device="cuda")
    M.moe_attention_tree(cache, wide[:, 2:6, :64], torch.from_numpy(first).cuda(), torch.from_numpy(p.lens).cuda(), outs[:, 1:5, 8:72], ws, 4, lse=lse)
    check_tree(p, q, first, p.lens, 4, outs[:, 1:5, 8:72].float().cpu().numpy(), lse.cpu().numpy())
    outs[:, 1:5, 8:72] = 7.0
    assert (outs == 7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinities(dtype):
    p = Paged([40, 40, 40, 40], 1, 64, 16, dtype)
    q = torch.ones(8, 2, 64, dtype=DT[dtype])
    first = firsts([2, 2, 2, 2])
    at = lambda s, j: (p.table[s, j // 16], j % 16, 0)  # noqa: E731
    for j in range(0, 39, 3):
        p.k[at(0, j)] = -np.inf
        p.v[at(0, j)] = 1.0
    for j in range(40):
        p.k[at(1, j)] = -np.inf
    p.k[at(2, 39)] = np.nan                # the second new token's own key: nothing to the first
    out, lse = attend_tree(p.cache(), q, first, p.lens, 2)
    assert np.isnan(out[5]).all() and np.isnan(lse[5]).all() and np.isfinite(out[4]).all()
    assert not out[2:4].any() and np.isneginf(lse[2:4]).all()
    p.k[at(2, 39)] = 0.0
    out[5], lse[5] = [x[5] for x in attend_tree(p.cache(), q, first, p.lens, 2)]
    check_tree(p, q, first, p.lens, 2, out, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nan_in_unseen_drafts(dtype):
    """A branch's NaN values reach no other branch."""
    p = Paged([70], 2, 64, 16, dtype)
    p.v[p.table[0, 69 // 16], 69 % 16] = np.nan
    p.k[p.table[0, 68 // 16], 68 % 16] = np.inf
    q, words = queries(6, 4, 64, dtype), np.array([1, 3, 5, 7, 16, 48], dtype=np.int64)
    out, lse = attend_tree(p.cache(), q, [0, 6], [70], 6, words)
    assert np.isfinite(out[:4]).all() and np.isnan(out[5]).any()
    ref = O.tree(np.nan_to_num(p.k), np.nan_to_num(p.v), p.table, q.float().numpy(), [0, 6], [70], 6, words, 0.125)
    assert np.abs(out[:4] - ref[0][:4]).max() < 2.0 ** -7 * np.abs(ref[0][:4]).max()


def test_one_token_equals_the_attention_of_one_token():
    """Same definition: one new token per sequence, with and without a window."""
    lens = [1, 17, 300, 64, 2000]
    for window in (0, 5, 100):
        p = Paged(lens, 2, 64, 16, "f32")
        q = queries(5, 8, 64, "f32")
        a, la = attend(p.cache(), q, lens, window=window)
        b, lb = attend_tree(p.cache(), q, firsts([1] * 5), lens, 1, window=window)
        # both within 2^-24 times (n + 80) of the definition, on values of size 1
        assert np.abs(a - b).max() < 2e-5 and np.abs(la - lb).max() < 2e-5


def test_results_do_not_change_and_graphs():
    p = Paged([1500, 17, 640], 2, 128, 16, "bf16")
    counts = [7, 3, 5]
    q, first, words = queries(15, 8, 128, "bf16"), firsts(counts), tree_words(counts)
    cache, qd = p.cache(), q.cuda()
    eager = attend_tree(cache, q, first, p.lens, 8, words)
    for _ in range(3):
        again = attend_tree(cache, q, first, p.lens, 8, words)
        assert np.array_equal(eager[0], again[0]) and np.array_equal(eager[1], again[1])
    dev = [torch.from_numpy(x).cuda() for x in (first, p.lens, words)]
    ws = torch.empty(M.moe_attention_tree_workspace_bytes(cache, 8, 8), dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(qd), torch.empty(15, 8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    M.moe_attention_tree(cache, qd, dev[0], dev[1], out, ws, 8, visible=dev[2], lse=lse, stream=s)
    s.synchronize()
    assert np.array_equal(eager[0], out.float().cpu().numpy())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        M.moe_attention_tree(cache, qd, dev[0], dev[1], out, ws, 8, visible=dev[2], lse=lse)
    # lengths, offsets and words are read when the graph runs
    for lens, counts in (([1500, 17, 640], [7, 3, 5]), ([1499, 3, 600], [1, 2, 8]), ([9, 17, 0], [4, 0, 2]), ([1500, 17, 640], [7, 3, 5])):
        first, words = firsts(counts), np.zeros(15, dtype=np.int64)
        words[:sum(counts)] = tree_words(counts, seed=sum(lens))
        for d, h in zip(dev, (first, np.array(lens, dtype=np.int32), words)):
            d.copy_(torch.from_numpy(h))
        out.fill_(float("nan"))
        lse.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        eager = attend_tree(cache, q, first, lens, 8, words)
        got = out.float().cpu().numpy()
        assert np.array_equal(eager[0], got, equal_nan=True) and np.array_equal(eager[1], lse.cpu().numpy(), equal_nan=True)
        check_tree(p, q, first, lens, 8, got, lse.cpu().numpy(), words)


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
    q, words = queries(5, 16, D, "bf16"), tree_words([5])
    out, lse = attend_tree(cache, q, [0, 5], [200], 5, words)
    check_tree(p, q, [0, 5], [200], 5, out, lse, words)
