"""Attention of one new token over a paged cache against the definition in 64 bits: lengths around tiles and pages, head groups and
dimensions of every kind, missing pages, caps, windows, biases, NaN wherever nothing may be read into a result."""
import numpy as np
import pytest
import torch

import paper_2205_10034_amd as M
from attention_util import DT, Paged, attend, check, queries

pytestmark = pytest.mark.gpu

RAGGED = [0, 1, 2, 15, 16, 17, 31, 33, 64, 127, 129, 300]


def run(lens, hq, hkv, D, page, dtype, layout="token_major", table=None, gain=2.0, pad=0, one_pool=False, spare_width=1, call_lens=None, **kw):
    print(lens, hq, hkv, D, page, dtype, layout, kw, flush=True)
    p = Paged(lens, hkv, D, page, dtype, layout, pad=pad, one_pool=one_pool, spare_width=spare_width)
    q = queries(len(lens), hq, D, dtype, gain=gain)
    call_lens = lens if call_lens is None else call_lens
    dev = {k: torch.from_numpy(v).cuda() if isinstance(v, np.ndarray) else v for k, v in kw.items()}
    out, lse = attend(p.cache(table), q, call_lens, **dev)
    check(p, q, call_lens, out, lse, table=table, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [1, 7, 16, 32, 100])
@pytest.mark.parametrize("layout", ["token_major", "head_major"])
def test_lengths_and_pages(page, layout, dtype):
    run(RAGGED, 4, 2, 64, page, dtype, layout)


@pytest.mark.parametrize("D,dtype", [(8, "bf16"), (24, "bf16"), (64, "bf16"), (72, "bf16"), (80, "bf16"), (96, "bf16"), (128, "bf16"), (136, "bf16"),
                                     (192, "bf16"), (256, "bf16"), (4, "f32"), (12, "f32"), (60, "f32"), (64, "f32"), (68, "f32"), (100, "f32"),
                                     (128, "f32"), (132, "f32"), (256, "f32")])
def test_head_dimensions(D, dtype):
    run([5, 70, 333], 6, 2, D, 16, dtype)
    run([0, 1, 200], 2, 2, D, 9, dtype, "head_major", softcap=20.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G", [1, 2, 5, 8, 15, 16, 17, 32, 33, 64])
def test_head_groups(G, dtype):
    run([3, 150, 0, 64], 2 * G, 2, 32, 16, dtype)
    run([90, 1], G, 1, 128, 32, dtype, "head_major")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", [[1], [4000], [70001], [1, 9000, 3, 0, 257], [0, 0, 0], [513] * 40])
def test_split_over_the_length(lens, dtype):
    run(lens, 8, 2, 64, 64, dtype)


def test_many_sequences():
    rng = np.random.default_rng(5)
    run(rng.integers(0, 60, 700).tolist(), 2, 1, 64, 16, "bf16")
    run([0] * 300 + [2000] + [1] * 300, 2, 2, 32, 16, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,D", [(8, 8, 64), (6, 6, 64), (5, 5, 64), (4, 1, 128), (48, 4, 64), (80, 2, 64), (8, 4, 256)])
def test_deals(hq, hkv, D, dtype):
    """The ways the work is dealt out: tables far wider than the lengths, all sequences short, some long, more sequences than
    workgroups, heads side by side or not."""
    rng = np.random.default_rng(hq)
    wide = dict(spare_width=300)
    run(rng.integers(0, 100, 200).tolist(), hq, hkv, D, 16, dtype, **wide)                      # all tiny
    run(rng.integers(0, 100, 200).tolist(), hq, hkv, D, 16, dtype, "head_major", window=3)
    run(rng.integers(0, 900, 12).tolist(), hq, hkv, D, 16, dtype, **wide)                       # short, fewer than workgroups
    run(rng.integers(0, 300, 150).tolist(), hq, hkv, D, 16, dtype)                              # short by the table, more than workgroups
    run(rng.integers(0, 300, 150).tolist(), hq, hkv, D, 16, dtype, **wide)                      # short, found out from the lengths
    run([2000] + rng.integers(0, 40, 80).tolist() + [1500], hq, hkv, D, 16, dtype, "head_major")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [1, 2, 16, 100, 129, 100000])
def test_window(window, dtype):
    run(RAGGED + [1000], 4, 2, 64, 16, dtype, window=window)
    run([2500], 4, 2, 64, 10, dtype, "head_major", window=window)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cap_and_distance_bias(dtype):
    slopes = np.array([0.5, 0.0, 0.03, 3.0, -0.01, 1e-4, 0.25, 0.125], dtype=np.float32)
    run(RAGGED, 8, 4, 64, 16, dtype, softcap=5.0, gain=8.0)
    run(RAGGED, 8, 4, 64, 16, dtype, slopes=slopes)
    run(RAGGED, 8, 4, 64, 16, dtype, slopes=slopes, softcap=30.0, window=50, scale=0.3)
    run([20000], 8, 1, 64, 16, dtype, slopes=slopes)
    run([40], 8, 4, 64, 16, dtype, scale=-0.2)
    run([40, 0], 8, 4, 64, 16, dtype, scale=0.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores(dtype):
    # scores of some hundreds: one key takes all the weight, the others underflow
    run([1, 40, 700], 4, 2, 64, 16, dtype, gain=300.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_missing_pages(dtype):
    lens = [100, 64, 300, 40, 20]
    p = Paged(lens, 2, 64, 16, dtype)
    table = p.table.copy()
    table[0, 2] = -1                       # in the middle
    table[1, :] = -5                       # all of them: nothing kept
    table[2, 0] = p.n_pages                # one past the pool
    table[2, 7:12] = 2 ** 31 - 1
    table[3, 2] = -2 ** 31                 # the last one
    run(lens, 4, 2, 64, 16, dtype, table=table)
    run(lens, 4, 2, 64, 16, dtype, table=table, window=20)
    run([700], 4, 2, 64, 16, dtype, table=np.full((1, 45), -1))


def test_lengths_outside_the_table():
    p_lens = [48, 32, 5]
    p = Paged(p_lens, 2, 64, 16, "bf16", spare_width=0)
    q = queries(3, 4, 64, "bf16")
    table = p.table
    full = [48, 1000, -3]                  # clamped to the three pages' 48 places (one of them missing), and to zero
    out, lse = attend(p.cache(), q, full)
    check(p, q, [48, 48, 0], out, lse, table=table)


def test_strides():
    run(RAGGED, 4, 2, 64, 16, "bf16", pad=8)
    run(RAGGED, 4, 2, 64, 16, "bf16", "head_major", pad=24, one_pool=True)
    run(RAGGED, 4, 2, 64, 7, "f32", one_pool=True, pad=4)
    # queries and outputs inside wider tensors
    p = Paged([5, 40, 130], 2, 64, 16, "bf16")
    q = queries(3, 4, 64, "bf16")
    wide = torch.full((3, 9, 72), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 2:6, :64] = q.cuda()
    outs = torch.full((3, 6, 80), 7.0, dtype=torch.bfloat16, device="cuda")
    cache = p.cache()
    ws = torch.empty(M.moe_attention_decode_workspace_bytes(cache, 4), dtype=torch.uint8, device="cuda")
    lse = torch.empty(3, 4, device="cuda")
    M.moe_attention_decode(cache, wide[:, 2:6, :64], torch.from_numpy(p.lens).cuda(), outs[:, 1:5, 8:72], ws, lse=lse)
    check(p, q, p.lens, outs[:, 1:5, 8:72].float().cpu().numpy(), lse.cpu().numpy())
    outs[:, 1:5, 8:72] = 7.0
    assert (outs == 7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinities(dtype):
    # keys of -infinity scores carry no weight; a sequence of nothing else has no output; a NaN key makes its own row NaN only
    p = Paged([40, 40, 40, 40], 1, 64, 16, dtype)
    q = torch.ones(4, 2, 64, dtype=DT[dtype])
    at = lambda s, j: (p.table[s, j // 16], j % 16, 0)
    for j in range(0, 40, 3):
        p.k[at(0, j)] = -np.inf
        p.v[at(0, j)] = 1.0
    for j in range(40):
        p.k[at(1, j)] = -np.inf
    p.k[at(2, 21)] = np.nan
    out, lse = attend(p.cache(), q, p.lens)
    assert np.isnan(out[2]).all() and np.isnan(lse[2]).all()
    assert not out[1].any() and np.isneginf(lse[1]).all()
    p.k[at(2, 21)] = 0.0
    out[2], lse[2] = [x[2] for x in attend(p.cache(), q, p.lens)]
    check(p, q, p.lens, out, lse)


def test_results_do_not_change():
    p = Paged([3000, 17, 0, 640], 2, 128, 16, "bf16")
    q = queries(4, 8, 128, "bf16")
    cache = p.cache()
    first = attend(cache, q, p.lens)
    for _ in range(3):
        again = attend(cache, q, p.lens)
        assert np.array_equal(first[0], again[0]) and np.array_equal(first[1], again[1])


def test_other_stream_and_graph():
    p = Paged([1500, 17, 0, 640], 2, 128, 16, "bf16")
    q = queries(4, 8, 128, "bf16")
    cache, qd, lens = p.cache(), q.cuda(), torch.from_numpy(p.lens).cuda()
    ws = torch.empty(M.moe_attention_decode_workspace_bytes(cache, 8), dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(qd), torch.empty(4, 8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    M.moe_attention_decode(cache, qd, lens, out, ws, lse=lse, stream=s)
    s.synchronize()
    check(p, q, p.lens, out.float().cpu().numpy(), lse.cpu().numpy())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        M.moe_attention_decode(cache, qd, lens, out, ws, lse=lse)
    # the lengths are read when the graph runs, not when it was captured
    for now in ([1500, 17, 0, 640], [3, 0, 0, 600], [1499, 17, 0, 1]):
        lens.copy_(torch.tensor(now, dtype=torch.int32))
        out.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        check(p, q, now, out.float().cpu().numpy(), lse.cpu().numpy())
        eager = attend(cache, q, now)
        assert np.array_equal(eager[0], out.float().cpu().numpy())


def test_places_beyond_32_bits():
    """Pages whose element offsets pass 2^31 and whose byte offsets pass 2^32: only four of a large pool's pages hold anything."""
    n_pages, page, hkv, D = 10000, 64, 16, 128       # 1.3e9 elements, 2.6 GB, in each pool
    far = [9999, 3, 8200, 9001]
    p = Paged([200], hkv, D, page, "bf16", spare_pages=0, spare_width=0)
    k = torch.full((2 * n_pages, page, hkv, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    v = torch.full((2 * n_pages, page, hkv, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    where = [2 * f for f in far]                      # up to page 19998: 2.6e9 elements
    for i, f in enumerate(where):
        k[f] = torch.from_numpy(p.k[p.table[0, i]]).cuda()
        v[f] = torch.from_numpy(p.v[p.table[0, i]]).cuda()
    cache = M.KVCache(k, v, torch.tensor([where], dtype=torch.int32, device="cuda"))
    q = queries(1, 16, D, "bf16")
    out, lse = attend(cache, q, [200])
    check(p, q, [200], out, lse)
