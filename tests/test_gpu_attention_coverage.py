"""Every kept place enters the decode attention once: long splits, ragged batches, windows, missing pages, and the kernels that read large
pools past the caches (chosen by the pool's size) for every type and head dimension."""
import numpy as np
import pytest
import torch

import paper_2205_10034_amd as M
from attention_coverage import Marked
from attention_util import DT, Paged, attend, check, queries

pytestmark = pytest.mark.gpu

RAGGED = np.random.default_rng(3).integers(0, 6000, 60).tolist()
LENS = {"long": [70001], "longest": [131071, 5, 0, 9000], "split": [20000, 1, 4097, 0, 513, 20000], "ragged": RAGGED, "one part more": [1025] * 33,
        "many": [40, 0, 1, 700] * 130, "many, one long": [17] * 300 + [12345] + [0] * 300}
ALL_LENGTHS = sorted(set(n for lens in LENS.values() for n in lens if n))
LARGE = 330.0   # megabytes of pool, beyond what is read through the caches


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,D", [(8, 2, 64), (1, 1, 128), (12, 4, 128), (40, 2, 256), (64, 1, 64), (3, 3, 64)])
@pytest.mark.parametrize("lens", LENS.values(), ids=LENS.keys())
def test_every_place_once(lens, hq, hkv, D, dtype):
    print(len(lens), hq, hkv, D, dtype, flush=True)
    m = Marked(lens, hkv, D, 16, dtype)
    m.check(hq)
    m.check(hq, window=1500)


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 64), ("f32", 128), ("f32", 256)])
@pytest.mark.parametrize("layout", ["token_major", "head_major"])
def test_every_place_of_a_large_pool_once(layout, dtype, D):
    print(layout, dtype, D, flush=True)
    lens = [30001, 0, 5, 1200, 64, 2000]
    missing = [(0, 3), (0, 1000), (3, 0), (4, 1)]
    for pool_mb, spare in ((LARGE, 1), (LARGE, 500)):
        m = Marked(lens, 2, D, 16, dtype, layout, pool_mb, missing, spare)
        for hq in (4, 40):
            m.check(hq)
            m.check(hq, window=700)


@pytest.mark.parametrize("dtype,D", [("bf16", 8), ("bf16", 64), ("bf16", 80), ("bf16", 128), ("bf16", 136), ("bf16", 256),
                                     ("f32", 12), ("f32", 64), ("f32", 100), ("f32", 128), ("f32", 132), ("f32", 256)])
def test_large_pools(dtype, D):
    """Random keys and values, sparsely in a pool beyond what is read through the caches; partial dimensions, splits, windows, caps."""
    print(dtype, D, flush=True)
    lens, hkv, page = [5000, 0, 1, 333, 16, 2048], 2, 16
    p = Paged(lens, hkv, D, page, dtype)
    n_pages = int(LARGE * 1e6 / (2 * page * hkv * D * p_bytes(dtype))) + p.n_pages
    where = torch.randperm(n_pages, generator=torch.Generator().manual_seed(5))[:p.n_pages]
    k = torch.full((n_pages, page, hkv, D), float("nan"), dtype=DT[dtype], device="cuda")
    v = k.clone()
    k[where.cuda()], v[where.cuda()] = (torch.from_numpy(x).to(DT[dtype]).cuda() for x in (p.k, p.v))
    compact = p.table.copy()
    compact[0, 7], compact[3, 2] = -1, p.n_pages   # two pages that are not there
    there = (compact >= 0) & (compact < p.n_pages)
    table = np.where(there, where.numpy()[np.where(there, compact, 0)], np.where(compact < 0, -1, n_pages)).astype(np.int32)
    cache = M.KVCache(k, v, torch.from_numpy(table).cuda())
    slopes = np.array([0.25, 0.0, 0.01, 1.0], dtype=np.float32)
    for hq, kw in ((4, {}), (34, {}), (4, dict(window=100)), (4, dict(softcap=20.0, slopes=slopes))):
        q = queries(len(lens), hq, D, dtype)
        dev = {n: torch.from_numpy(x).cuda() if isinstance(x, np.ndarray) else x for n, x in kw.items()}
        out, lse = attend(cache, q, lens, **dev)
        check(p, q, lens, out, lse, table=compact, **kw)


def p_bytes(dtype):
    return 2 if dtype == "bf16" else 4
