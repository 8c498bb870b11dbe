"""Host-only: a workspace that was sized once, for the largest call, is enough for every smaller one."""
import ctypes as C
import random

import pytest

from paper_2205_10034_amd import drafts as D
from paper_2205_10034_amd import logprobs as P
from test_attention_abi import FAKE, ROWS, cache

T_STEPS = list(range(1, 300)) + [300, 511, 512, 513, 575, 576, 600, 1000, 1023, 1024, 1025, 1500, 2047, 2048, 2049, 3000, 8192, 16384]


@pytest.mark.parametrize("V", [1, 100, 2000, 16000, 17000, 50001, 65000, 65535, 66000, 128000, 250000, 262144, 1 << 20])
@pytest.mark.parametrize("K", [0, 1, 20, 64])
def test_fewer_rows(V, K):
    if K > V:
        return
    sizes = [P.lib().moe_token_logprobs_workspace_bytes(T, V, K) for T in T_STEPS]
    assert all(a <= b for a, b in zip(sizes, sizes[1:])), [(T, a, b) for T, a, b in zip(T_STEPS, sizes, sizes[1:]) if a > b][:5]


def test_shorter_rows_and_fewer_alternatives():
    L, rng = P.lib(), random.Random(5)
    for _ in range(4000):
        T, V, K = rng.choice(T_STEPS), int(2 ** rng.uniform(0, 20)), rng.choice([0, 1, 5, 64])
        t, v, k = rng.randint(0, T), rng.randint(1, V), rng.randint(0, K)
        if K <= V and k <= v:
            assert L.moe_token_logprobs_workspace_bytes(t, v, k) <= L.moe_token_logprobs_workspace_bytes(T, V, K), (t, v, k, T, V, K)


def test_fewer_drafts():
    """Also across the numbers of rows at which another kernel runs."""
    L, rng, dips = D.lib(), random.Random(7), []
    shapes = [(dict(n_seqs=s, n_kv_heads=hkv, head_dim=d, table_width=w, page_size=16, dtype=dtype, page_stride=1 << 20, token_stride=1 << 12, head_stride=256), hkv * G)
              for s in (1, 3, 100, 1000) for hkv in (1, 2, 5, 8, 16, 100) for G in (1, 3, 4, 16, 40) for d in (64, 128, 256) for w in (1, 30, 5000) for dtype in (0, 1)]
    for kw, hq in rng.sample(shapes, 400) + [(dict(n_seqs=64, n_kv_heads=1, head_dim=256, table_width=4096, page_size=16), 4)]:
        c = cache(**kw)
        sizes = [L.moe_attention_tree_workspace_bytes(C.byref(c), hq, n) for n in range(1, 65)]
        assert min(sizes) >= 256
        dips += [(kw, hq, n, a, b) for n, a, b in zip(range(1, 65), sizes, sizes[1:]) if a > b]
    assert not dips, (len(dips), dips[:3])


def test_what_is_too_small_is_still_refused():
    L, c = D.lib(), cache(n_kv_heads=1, head_dim=256, table_width=4096, n_seqs=64)
    need = L.moe_attention_tree_workspace_bytes(C.byref(c), 4, 33)
    opt = D._Options(scale=1.0, softcap=0.0, window=0, sinks=0, slopes=None)
    assert L.moe_attention_tree(C.byref(c), 4, 5, 33, C.byref(ROWS()), FAKE, FAKE, None, C.byref(opt), C.byref(ROWS(2 * FAKE)), None, FAKE, need - 1, None) == 3
    L = P.lib()
    for T, V, K in ((300, 128000, 0), (1, 1 << 20, 0), (1025, 50001, 5)):
        need = L.moe_token_logprobs_workspace_bytes(T, V, K)
        assert L.moe_token_logprobs(1, T, V, FAKE, V, 1.0, FAKE, FAKE, FAKE, None, K, FAKE, FAKE, FAKE, need - 1, None) == 3
