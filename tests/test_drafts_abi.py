"""Host-only checks of a step of drafted tokens and of the log-probabilities: the oracle's own pins, refusals of the C ABI and of the
binding, and which rows, places and positions are a token's, compiled for the host."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest
import torch

import paper_2205_10034_amd as M
from oracle import attention_oracle as A
from oracle import drafts_oracle as O
from paper_2205_10034_amd import attention as B
from paper_2205_10034_amd import drafts as D
from paper_2205_10034_amd import logprobs as P
from test_attention_abi import FAKE, ROWS, cache

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ref = lambda s: C.byref(s) if s is not None else None  # noqa: E731
OPT = lambda **kw: D._Options(**{**dict(scale=0.125, softcap=0.0, window=0, sinks=0, slopes=None), **kw})  # noqa: E731


# ---- oracle ------------------------------------------------------------------------------------------

def small_cache(seed=0):
    rng = np.random.default_rng(seed)
    return rng.standard_normal((6, 4, 2, 8)), rng.standard_normal((6, 4, 2, 8)), np.array([[3, 0, 4], [5, 1, 2]])


def test_oracle_chain_is_the_attention_of_one_token_again_and_again():
    k, v, table = small_cache()
    q = np.random.default_rng(1).standard_normal((5, 4, 8))
    slopes = [0.1, 0.0, 0.3, -0.2]
    for window in (0, 3):
        out, lse, *_ = O.tree(k, v, table, q, [0, 3, 5], [10, 7], 3, None, 0.3, 4.0, window, 0, slopes)
        for s, first, n, length in ((0, 0, 3, 10), (1, 3, 2, 7)):
            for i in range(n):
                o, l, *_ = A.decode(k, v, table[s:s + 1], q[first + i:first + i + 1], [length - n + 1 + i], 0.3, 4.0, window, slopes)
                assert np.allclose(out[first + i], o[0]) and np.allclose(lse[first + i], l[0])


def test_oracle_tree_branches_are_chains_of_their_own():
    """A token of a tree has what a chain of its ancestors gives it, their keys and values moved up behind the cache."""
    k, v, table = small_cache(2)
    q = np.random.default_rng(3).standard_normal((5, 4, 8))
    words = np.array([0b1, 0b11, 0b101, 0b1101, 0b10011], dtype=np.int64)       # 0 - 1 - 4 and 0 - 2 - 3
    for window, sinks in ((0, 0), (3, 0), (3, 2)):
        out, lse, *_ = O.tree(k, v, table[:1], q, [0, 5], [11], 5, words, 0.3, window=window, sinks=sinks, slopes=[0.5, 0.1, 0.0, 1.0])
        for i, path in ((3, [0, 2, 3]), (4, [0, 1, 4]), (1, [0, 1])):
            (k2, v2), lens = O.compact([k, v], table[:1], [6], [path])
            o, l, *_ = O.tree(k2, v2, table[:1], q[path], [0, len(path)], lens, 5, None, 0.3, window=window, sinks=sinks, slopes=[0.5, 0.1, 0.0, 1.0])
            assert np.allclose(out[i], o[-1]) and np.allclose(lse[i], l[-1])


def test_oracle_tree_limits():
    k, v, table = small_cache(4)
    q = np.ones((6, 2, 8))
    out, lse, *rest = O.tree(k, v, table, q, [0, 2, 4], [2, 1], 2, np.zeros(6, dtype=np.int64), 1.0)
    assert not out[:2].any() and np.isneginf(lse[:4]).all() and np.isnan(out[4:]).all()      # nothing cached, nothing seen
    out, lse, *rest = O.tree(k, v, table, q, [0, 1, 1], [5, 9], 4, None, 1.0, window=1)
    assert rest[-1].tolist() == [1, 0, 0, 0, 0, 0] and np.allclose(out[0], np.broadcast_to(v[0, 0][:, None], (2, 1, 8))[:, 0])   # its own place, the fifth
    assert O.tree(k, v, table, q, [0, 1, 1], [9, 9], 4, None, 1.0, window=1, sinks=3)[-1][0] == 4
    assert O.cut([0, 9, 2], [7, -3], 6, 4, 12) == [(0, 4, 3, 7), (6, 0, 0, 0)]


def test_oracle_pages():
    p = O.Pages(np.full((3, 4), -1), np.zeros(6), 4)
    assert p.reserve([9, -1, 4], 0) == 0 and p.table == [[0, 1, 2, -1], [-1] * 4, [3, -1, -1, -1]]
    lens = [9, -1, 4]
    assert p.fork([0], [1], lens) == ([(2, 4, 1)], 0) and p.table[1] == [0, 1, 4, -1] and lens == [9, 9, 4] and p.refs == [2, 2, 1, 1, 1, 0]
    p.release([4, 9, -1])
    assert p.refs == [2, 1, 0, 0, 1, 0] and p.consistent()
    assert p.reserve([16, 9, -1], 5) == 1 and p.table[0] == [0, 2, 3, 5] and p.reserve([-1, 16, -1], 0) == 1 and p.table[1] == [0, 1, 4, -1]


def test_oracle_forks_that_are_left_out():
    p = O.Pages(np.full((5, 3), -1), np.zeros(20), 4)
    lens = [9, 5, 2, 7, 1]
    p.reserve(lens, 0)
    p.fork([0, 1, 2, 4], [3, 3, 4, 0], lens)          # 3 twice; 4 and 0 are sources
    assert lens == [9, 5, 2, 9, 1] and p.consistent() and p.table[3][:2] == p.table[0][:2]


def test_oracle_compact_reads_before_it_writes():
    k = np.arange(6 * 4 * 2 * 8, dtype=float).reshape(6, 4, 2, 8)
    table = np.array([[3, 0, 4], [5, -1, 2]])
    (new,), lens = O.compact([k], table, [2, 3], [[1, 0, 5, -1], [2, 5, 1, 0]])
    assert np.array_equal(new[3, 2], k[3, 3]) and np.array_equal(new[3, 3], k[3, 2]) and np.array_equal(new[0, 0], k[0, 3]) and lens == [5, 7]
    assert np.array_equal(new[5, 3], k[5, 3]) and np.array_equal(new[5, :3], k[5, :3]) and np.array_equal(new[2], k[2])


def test_oracle_logprobs_against_a_library():
    rng = np.random.default_rng(0)
    x, ids = rng.standard_normal((3, 10)), [1, 2, -1]
    z = torch.from_numpy(x).requires_grad_(True)
    lp = torch.log_softmax(z * 0.5, 1)
    ent = -(lp.exp() * lp).sum(1)
    logp, lse, h, order, top, p = O.logprobs(x, ids, 0.5, 3)
    assert np.allclose(logp, [lp[0, 1].item(), lp[1, 2].item(), 0]) and np.allclose(h, ent.detach()) and np.allclose(lse, torch.logsumexp(z * 0.5, 1).detach())
    assert np.array_equal(order, torch.topk(lp, 3, 1)[1]) and np.allclose(top, torch.topk(lp, 3, 1)[0].detach())
    (2 * lp[0, 1] + 3 * lp[1, 2] + (ent * torch.tensor([1.0, 2.0, 3.0])).sum() + 0.7 * torch.logsumexp(z * 0.5, 1).sum()).backward()
    d, _ = O.logprobs_gradient(x, ids, 0.5, [2, 3, 4], [1, 2, 3], [0.7] * 3)
    assert np.allclose(d, z.grad)


def test_oracle_logprobs_limits():
    x = np.array([[-np.inf] * 3, [1, -np.inf, -np.inf], [0, np.nan, 9], [np.inf, 0, 1], [2, 2, 2]])
    logp, lse, h, order, top, p = O.logprobs(x, [0, 1, 2, 0, 1], 1.0, 3)
    assert np.isneginf(lse[0]) and np.isneginf(logp[0]) and h[0] == 0 and not p[0].any()
    assert lse[1] == 1 and np.isneginf(logp[1]) and h[1] == 0 and top[1, 0] == 0 and order[1].tolist() == [0, 1, 2]
    assert np.isnan([lse[2], lse[3], logp[2], h[3], top[2, 0], top[3, 1]]).all() and order[2].tolist() == [2, 0, 1] and order[3].tolist() == [0, 2, 1]
    assert order[4].tolist() == [0, 1, 2] and np.allclose(h[4], np.log(3))
    d, _ = O.logprobs_gradient(x, [0, 0, -1, 1, 1], 1.0, [1.0] * 5)
    assert not d[:3].any() and np.isnan(d[3]).all() and np.allclose(d[4], [-1 / 3, 2 / 3, -1 / 3])


# ---- refusals ------------------------------------------------------------------------------------------

BAD_CACHES = [dict(dtype=2), dict(head_dim=60), dict(head_dim=264), dict(n_kv_heads=0), dict(page_size=0), dict(n_seqs=-1), dict(table_width=2 ** 28), dict(n_pages=2 ** 31),
              dict(token_stride=12), dict(k=FAKE + 8), dict(v=None), dict(page_table=None)]


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_bad_caches_are_refused(bad):
    L, c, r = D.lib(), cache(**bad), ROWS()
    assert L.moe_attention_tree_workspace_bytes(ref(c), 4, 8) == 0 and L.moe_kv_pages_workspace_bytes(ref(c)) == 0
    assert L.moe_attention_tree(ref(c), 4, 5, 8, ref(r), FAKE, FAKE, None, ref(OPT()), ref(ROWS(2 * FAKE)), None, FAKE, 1 << 40, None) == 1
    assert L.moe_kv_compact(ref(c), FAKE, 4, FAKE, None, None) == 1 and L.moe_kv_release(ref(c), FAKE, FAKE, None) == 1
    assert L.moe_kv_fork(ref(c), FAKE, 1, FAKE, FAKE, FAKE, None, FAKE, 1 << 40, None) == 1
    assert L.moe_kv_reserve(ref(c), FAKE, FAKE, 1, None, FAKE, 1 << 40, None) == 1
    assert len(L.moe_last_error()) > 0


def test_tree_attention_refuses():
    L, c, x, y = D.lib(), cache(), ROWS(), ROWS(2 * FAKE)
    need = L.moe_attention_tree_workspace_bytes(ref(c), 4, 8)
    assert need >= 256 and need % 256 == 0
    for hq, n in ((0, 8), (3, 8), (-2, 8), (1 << 18, 8), (4, 0), (4, 65), (4, -1)):
        assert L.moe_attention_tree_workspace_bytes(ref(c), hq, n) == 0

    def call(c=c, hq=4, T=5, n_max=8, q=x, first=FAKE, lens=FAKE, opt=OPT(), out=y, ws=FAKE, n=need):
        return L.moe_attention_tree(ref(c), hq, T, n_max, ref(q), first, lens, None, ref(opt), ref(out), None, ws, n, None)

    for bad in (dict(c=None), dict(hq=0), dict(hq=3), dict(T=-1), dict(n_max=0), dict(n_max=65), dict(q=None), dict(q=ROWS(None)), dict(q=ROWS(FAKE + 2)), dict(q=ROWS(t=100)),
                dict(first=None), dict(lens=None), dict(opt=None), dict(opt=OPT(scale=float("nan"))), dict(opt=OPT(softcap=-1.0)), dict(opt=OPT(softcap=float("inf"))),
                dict(opt=OPT(window=-1)), dict(opt=OPT(sinks=-1)), dict(out=None), dict(out=ROWS(2 * FAKE, 128, 63)), dict(out=x)):
        assert call(**bad) == 1, bad
    assert call(T=2 ** 24) == 2                                      # times 4 heads
    for bad in (dict(ws=None), dict(ws=FAKE + 16), dict(n=need - 1)):
        assert call(**bad) == 3, bad
    assert call(c=cache(n_seqs=0), q=None) == 0 and call(T=0, q=None) == 0


def test_pages_refuse():
    L, c = D.lib(), cache()
    need = L.moe_kv_pages_workspace_bytes(ref(c))
    assert need >= 256 and need % 256 == 0
    for bad in (dict(width=0), dict(width=65), dict(base=None), dict(keep=None), dict(new=FAKE)):
        kw = {**dict(base=FAKE, width=4, keep=2 * FAKE, new=None), **bad}
        assert L.moe_kv_compact(ref(c), kw["base"], kw["width"], kw["keep"], kw["new"], None) == 1, bad
    assert L.moe_kv_compact(ref(cache(n_seqs=0)), None, 4, None, None, None) == 0
    assert L.moe_kv_compact(ref(cache(n_seqs=2 ** 24, n_kv_heads=2)), FAKE, 4, 2 * FAKE, None, None) == 2
    assert L.moe_kv_release(ref(c), None, FAKE, None) == 1 and L.moe_kv_release(ref(c), FAKE, None, None) == 1
    assert L.moe_kv_release(ref(cache(n_seqs=0)), FAKE, None, None) == 0

    def fork(n=1, refs=FAKE, src=FAKE, dst=FAKE, lens=FAKE, ws=FAKE, size=need):
        return L.moe_kv_fork(ref(c), refs, n, src, dst, lens, None, ws, size, None)

    for bad in (dict(n=-1), dict(n=4), dict(refs=None), dict(src=None), dict(dst=None), dict(lens=None)):
        assert fork(**bad) == 1, bad
    assert fork(n=0, src=None, dst=None, lens=None) == 0

    def reserve(refs=FAKE, lens=FAKE, more=1, ws=FAKE, size=need):
        return L.moe_kv_reserve(ref(c), refs, lens, more, None, ws, size, None)

    for bad in (dict(refs=None), dict(lens=None), dict(more=-1)):
        assert reserve(**bad) == 1, bad
    for call in (fork, reserve):
        for bad in (dict(ws=None), dict(ws=FAKE + 16), dict(size=need - 1)):
            assert call(**bad) == 3, bad


def test_logprobs_refuse():
    L = P.lib()
    need = L.moe_token_logprobs_workspace_bytes(5, 100, 8)
    assert need >= 256 and need % 256 == 0
    for T, V, K in ((-1, 100, 8), (5, 0, 0), (5, 100, -1), (5, 100, 65), (5, 7, 8)):
        assert L.moe_token_logprobs_workspace_bytes(T, V, K) == 0

    def call(dtype=1, T=5, V=100, x=FAKE, stride=100, scale=1.0, ids=FAKE, logp=FAKE, K=8, top=FAKE, toplp=FAKE, ws=FAKE, n=need):
        return L.moe_token_logprobs(dtype, T, V, x, stride, scale, ids, logp, FAKE, None, K, top, toplp, ws, n, None)

    for bad in (dict(dtype=2), dict(T=-1), dict(V=0), dict(x=None), dict(x=FAKE + 1), dict(dtype=0, x=FAKE + 2), dict(stride=-1), dict(scale=0.0), dict(scale=-1.0),
                dict(scale=float("nan")), dict(scale=float("inf")), dict(ids=None), dict(K=65), dict(K=-1), dict(V=7), dict(top=None), dict(toplp=None)):
        assert call(**bad) == 1, bad
    assert call(T=2 ** 30) == 2
    for bad in (dict(ws=None), dict(ws=FAKE + 16), dict(n=need - 1)):
        assert call(**bad) == 3, bad
    assert call(T=0, x=None) == 0

    def grad(dtype=1, T=5, V=100, x=FAKE, stride=100, scale=1.0, ids=FAKE, lse=FAKE, d_logp=FAKE, ent=FAKE, d_ent=FAKE, d_x=2 * FAKE, d_stride=100):
        return L.moe_token_logprobs_backward(dtype, T, V, x, stride, scale, ids, lse, d_logp, ent, d_ent, None, d_x, d_stride, None)

    for bad in (dict(dtype=2), dict(T=-1), dict(V=0), dict(x=None), dict(x=FAKE + 1), dict(stride=-1), dict(scale=0.0), dict(ids=None), dict(lse=None), dict(ent=None),
                dict(d_x=None), dict(d_x=2 * FAKE + 1), dict(d_stride=99), dict(d_x=FAKE, d_stride=101), dict(d_stride=-1)):
        assert grad(**bad) == 1, bad
    assert grad(T=2 ** 30) == 2 and grad(T=0, x=None) == 0


def test_binding_refuses():
    with pytest.raises(ValueError, match="device tensors"):
        M.moe_token_logprobs(torch.zeros(2, 5), None, torch.zeros(256, dtype=torch.uint8))
    with pytest.raises(ValueError, match="bfloat16"):
        M.moe_token_logprobs(torch.zeros(2, 5, dtype=torch.float16), None, torch.zeros(256, dtype=torch.uint8))
    with pytest.raises(ValueError, match="contiguous"):
        P._matrix(torch.zeros(5, 2).t(), "logits", None, torch.float32, -1)
    with pytest.raises(ValueError, match="matrix"):
        P._matrix(torch.zeros(5), "logits", None, torch.float32, -1)
    with pytest.raises(ValueError, match="shape"):
        P._matrix(torch.zeros(5, 3), "d_logits", (5, 2), torch.float32, -1)
    for T, V, K in ((-1, 5, 0), (5, 0, 0), (5, 5, 6)):
        with pytest.raises(M.MoEError):
            M.moe_token_logprobs_workspace_bytes(T, V, K)
    with pytest.raises(ValueError, match="int32"):
        M.moe_token_logprobs_workspace_bytes(2 ** 31, 5, 0)
    assert [D._count(n) for n in (0, 5, 2 ** 31 - 1, 2 ** 31, 2 ** 80, -1, -2 ** 80)] == [0, 5, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1, -1, -1]


# ---- rows, places and positions, on the host ----------------------------------------------------------------

def test_drafts_on_the_host(tmp_path):
    src, exe = tmp_path / "drafts.cpp", tmp_path / "drafts"
    src.write_text("""#include "draft_tokens.h"
#include <cassert>
#include <initializer_list>
using namespace moesys;
int main() {
  const int far[] = {-2147483647 - 1, -5, 0, 1, 3, 7, 64, 100, 2147483647};
  for (int from : far) for (int to : far) for (int T : {1, 5, 100}) for (int most : {1, 8, 64}) for (int len : far) for (int cap : {0, 5, 2147483647}) {
    const Drafts d = drafts_of(from, to, T, most, len, cap);
    assert(d.first >= 0 && d.first <= T && d.n >= 0 && d.n <= most && d.first + d.n <= T && d.len >= 0 && d.len <= cap && d.base >= 0 && d.base <= d.len);
    assert(d.len < d.n ? d.base == 0 : d.base + d.n == d.len);
  }
  assert(drafts_of(2, 7, 9, 64, 40, 100).first == 2 && drafts_of(2, 7, 9, 64, 40, 100).n == 5 && drafts_of(2, 7, 9, 64, 40, 100).base == 35);
  for (int n = 1; n <= 64; ++n) {
    assert(bits_set(drafts_mask(n)) == n);
    for (int i = 0; i < n; ++i) {
      assert(seen_drafts(false, 0, i, n) == drafts_mask(i + 1) && draft_depth(seen_drafts(false, 0, i, n), i) == i);
      assert(seen_drafts(true, ~0ull, i, n) == drafts_mask(n) && draft_depth(~0ull & drafts_mask(n), i) == n - 1 && draft_depth(0, i) == 0);
    }
  }
  assert(in_window(9, 9, 9, 1, 0) && !in_window(9, 8, 8, 1, 0) && in_window(9, 2, 2, 1, 3) && in_window(9, 0, 0, 0, 0) && in_window(3, 9, 9, 1, 0));
  assert(!in_window(2147483647, 0, 0, 2147483647, 0) && in_window(2147483647, 1, 1, 2147483647, 0));
}""")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I" + os.path.join(ROOT, "paper_2205_10034_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    subprocess.run([str(exe)], check=True)
