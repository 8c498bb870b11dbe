"""Host-only checks of the attention half: the oracle's own pins, refusals of the C ABI and of the binding, and the arithmetic of
places, compiled for the host."""
import ctypes as C
import math
import os
import subprocess

import numpy as np
import pytest
import torch

import paper_2205_10034_amd as M
from oracle import attention_oracle as A
from paper_2205_10034_amd import attention as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x100000


# ---- oracle ------------------------------------------------------------------------------------------

def test_oracle_rotary_turns_by_the_angle():
    x = np.zeros((2, 1, 6))
    x[:, 0, 0], x[:, 0, 4] = 1.0, 5.0
    y = A.rotary(x, [[1, 3]], [0.5, 2.0], [2])
    for t, p in enumerate((1, 3)):
        assert np.allclose(y[t, 0], [math.cos(0.5 * p), 0, math.sin(0.5 * p), 0, 5, 0])
    y = A.rotary(x, [[1, 3]], [0.5, 2.0], [2], interleaved=True)
    assert np.allclose(y[1, 0], [math.cos(1.5), math.sin(1.5), 0, 0, 5, 0])
    rng = np.random.default_rng(0)
    x, pos, f = rng.standard_normal((4, 3, 12)), rng.integers(0, 99, (3, 4)), rng.random(6)
    y = A.rotary(x, pos, f, [1, 2, 3])
    assert np.allclose(A.rotary(y, pos, f, [1, 2, 3], inverse=True), x) and np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
    assert np.allclose(y[2, :, [3, 9]], A.rotary(x, [pos[2]], f, [6])[2, :, [3, 9]])  # pair 3 turns with the third axis


def test_oracle_decode_is_a_softmax():
    rng = np.random.default_rng(1)
    k, v, q = rng.standard_normal((5, 4, 2, 8)), rng.standard_normal((5, 4, 2, 8)), rng.standard_normal((1, 4, 8))
    table = np.array([[3, 0, 4]])
    out, lse, *_ = A.decode(k, v, table, q, [10], 0.3)
    kk, vv = np.concatenate([k[3], k[0], k[4]])[:10], np.concatenate([v[3], v[0], v[4]])[:10]
    want = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q[:, :, None]), torch.from_numpy(kk.transpose(1, 0, 2).repeat(2, 0)[None]),
                                                            torch.from_numpy(vv.transpose(1, 0, 2).repeat(2, 0)[None]), scale=0.3)[0, :, 0].numpy()
    assert np.allclose(out[0], want) and np.allclose(np.exp(lse[0, 0]), np.exp(0.3 * kk[:, 0] @ q[0, 0]).sum())
    # a window of one is the last value; a missing page drops its keys; a strong bias leaves the last
    assert np.allclose(A.decode(k, v, table, q, [10], 0.3, window=1)[0][0, 3], vv[9, 1])
    less = A.decode(k, v, np.array([[3, -1, 4]]), q, [10], 0.3)[0]
    keep = [0, 1, 2, 3, 8, 9]
    w = np.exp(0.3 * kk[keep, 0] @ q[0, 0])
    assert np.allclose(less[0, 0], (w / w.sum()) @ vv[keep, 0])
    assert np.allclose(A.decode(k, v, table, q, [10], 0.3, slopes=[1e4] * 4)[0][0, 0], vv[9, 0])
    out, lse, *_ = A.decode(k, v, table, q, [0], 0.3)
    assert not out.any() and np.isneginf(lse).all()


# ---- refusals ------------------------------------------------------------------------------------------

def cache(**kw):
    c = dict(k=FAKE, v=FAKE, page_table=FAKE, n_pages=10, page_stride=16 * 2 * 64, token_stride=128, head_stride=64, page_size=16, n_seqs=3,
             table_width=4, n_kv_heads=2, head_dim=64, dtype=1)
    c.update(kw)
    return B._Cache(**c)


def rotary(pairs=(32,), **kw):
    d = dict(head_dim=64, rot_dim=64, interleaved=0, n_axes=len(pairs), freqs=FAKE)
    d.update(kw)
    return B._RotarySpec(axis_pairs=(C.c_int32 * 3)(*(list(pairs) + [0] * (3 - len(pairs)))), **d)


ROWS = lambda data=FAKE, t=128, h=64: B._HeadRows(data, t, h)
OPT = lambda **kw: B._Options(**{**dict(scale=0.125, softcap=0.0, window=0, slopes=None), **kw})


@pytest.mark.parametrize("bad", [dict(dtype=2), dict(head_dim=0), dict(head_dim=60), dict(head_dim=264), dict(head_dim=2, dtype=0), dict(n_kv_heads=0),
                                 dict(page_size=0), dict(n_seqs=-1), dict(table_width=-1), dict(table_width=2 ** 28), dict(n_pages=-1),
                                 dict(n_pages=2 ** 31), dict(page_stride=-8), dict(token_stride=12), dict(head_stride=2, dtype=0), dict(k=FAKE + 8),
                                 dict(v=None), dict(page_table=None)])
def test_bad_caches_are_refused(bad):
    L, c = B.lib(), cache(**bad)
    assert L.moe_kv_cache_check(C.byref(c)) == 1 and len(L.moe_last_error()) > 0
    assert L.moe_attention_decode_workspace_bytes(C.byref(c), 4) == 0
    r = ROWS()
    assert L.moe_attention_decode(C.byref(c), 4, C.byref(r), FAKE, C.byref(OPT()), C.byref(r), None, FAKE, 1 << 40, None) == 1
    assert L.moe_kv_append(C.byref(c), 1, C.byref(r), C.byref(r), None, FAKE, None, None, 0, None, None, None) == 1


@pytest.mark.parametrize("bad", [dict(head_dim=1), dict(head_dim=258), dict(rot_dim=0), dict(rot_dim=63), dict(rot_dim=66), dict(interleaved=2), dict(n_axes=0),
                                 dict(n_axes=4), dict(pairs=(31,)), dict(pairs=(40, -8)), dict(pairs=(16, 8, 9)), dict(freqs=None)])
def test_bad_rotary_positions_are_refused(bad):
    L, r, x = B.lib(), rotary(**bad), ROWS()
    assert L.moe_rotary(C.byref(r), 1, 3, 2, C.byref(x), FAKE, C.byref(ROWS(FAKE * 2)), 0, None) == 1 and len(L.moe_last_error()) > 0
    assert L.moe_kv_append(C.byref(cache()), 3, C.byref(x), C.byref(x), None, FAKE, C.byref(r), FAKE, 0, None, None, None) == 1


def test_rotary_refuses():
    L, r, x, y = B.lib(), rotary(), ROWS(), ROWS(FAKE * 2)
    call = lambda dtype=1, T=3, H=2, x=x, pos=FAKE, out=y, inv=0: L.moe_rotary(C.byref(r), dtype, T, H, C.byref(x) if x else None, pos, C.byref(out) if out else None, inv, None)
    assert L.moe_rotary(None, 1, 3, 2, C.byref(x), FAKE, C.byref(y), 0, None) == 1
    for bad in (dict(dtype=5), dict(T=-1), dict(H=0), dict(x=None), dict(x=ROWS(None)), dict(pos=None), dict(out=None), dict(out=ROWS(None)), dict(inv=2),
                dict(out=ROWS(FAKE, 256, 64)), dict(H=2 ** 31 - 1)):
        assert call(**bad) == 1, bad
    assert call(T=0, x=None) == 0


def test_append_refuses():
    L, c, x, y, r = B.lib(), cache(), ROWS(), ROWS(FAKE * 2), rotary()
    ref = lambda s: C.byref(s) if s is not None else None

    def call(T=3, k=x, v=x, seq=None, at=FAKE, r=None, pos=None, hq=0, q=None, qo=None):
        return L.moe_kv_append(C.byref(c), T, ref(k), ref(v), seq, at, ref(r), pos, hq, ref(q), ref(qo), None)

    assert L.moe_kv_append(None, 1, ref(x), ref(x), None, FAKE, None, None, 0, None, None, None) == 1
    for bad in (dict(T=-1), dict(k=None), dict(v=None), dict(k=ROWS(None)), dict(at=None), dict(T=4), dict(q=x, qo=y, hq=2), dict(r=r, q=x, qo=y, hq=0),
                dict(r=r, q=x, hq=2), dict(r=r, q=x, qo=ROWS(None), hq=2), dict(r=rotary((16, 16))), dict(r=rotary(head_dim=128)),
                dict(r=r, q=x, qo=ROWS(FAKE, 64, 64), hq=2)):
        assert call(**bad) == 1, bad
    assert call(T=0, k=None) == 0


def test_attention_refuses():
    L, c, x, y = B.lib(), cache(), ROWS(), ROWS(FAKE * 2)
    ref = lambda s: C.byref(s) if s is not None else None
    need = L.moe_attention_decode_workspace_bytes(ref(c), 4)
    assert need >= 256 and need % 256 == 0

    def call(c=c, hq=4, q=x, lens=FAKE, opt=OPT(), out=y, ws=FAKE, n=need):
        return L.moe_attention_decode(ref(c), hq, ref(q), lens, ref(opt), ref(out), None, ws, n, None)

    for bad in (dict(c=None), dict(hq=0), dict(hq=3), dict(hq=-2), dict(q=None), dict(q=ROWS(None)), dict(q=ROWS(FAKE + 2)), dict(q=ROWS(t=100)), dict(lens=None),
                dict(opt=None), dict(opt=OPT(scale=float("nan"))), dict(opt=OPT(softcap=-1.0)), dict(opt=OPT(softcap=float("inf"))),
                dict(opt=OPT(window=-1)), dict(out=None), dict(out=ROWS(FAKE, 128, 63))):
        assert call(**bad) == 1, bad
    for bad in (dict(ws=None), dict(ws=FAKE + 16), dict(n=need - 1)):
        assert call(**bad) == 3, bad
    assert call(c=cache(n_seqs=0), q=None) == 0


def test_binding_refuses():
    k, table = torch.zeros(4, 16, 2, 64), torch.zeros(2, 2, dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensors"):
        M.KVCache(k, k, table)
    with pytest.raises(ValueError, match="layout"):
        M.KVCache(k, k, table, layout="rows")
    with pytest.raises(ValueError, match="one shape"):
        M.KVCache(k, k[:, :8], table)
    with pytest.raises(ValueError, match="contiguous"):
        M.KVCache(k.transpose(1, 3), k.transpose(1, 3), table)
    with pytest.raises(ValueError, match="page_table"):
        M.KVCache(k, k, table.long())
    with pytest.raises(ValueError, match="float64"):
        M.Rotary(64, torch.zeros(32))
    with pytest.raises(ValueError, match="device tensors"):
        M.Rotary(64, torch.zeros(32, dtype=torch.float64))
    x = torch.zeros(3, 2, 64)
    with pytest.raises(ValueError, match="shape"):
        B._rows(x, "x", (3, 2, 32), torch.float32, -1)
    with pytest.raises(ValueError, match="bfloat16"):
        B._rows(x, "x", (3, 2, 64), torch.bfloat16, -1)
    with pytest.raises(ValueError, match="contiguous"):
        B._rows(x.transpose(1, 2), "x", (3, 64, 2), torch.float32, -1)
    with pytest.raises(ValueError, match="int32"):
        B._vector(torch.zeros(3), "seq_lens", torch.int32, (3,), -1)
    with pytest.raises(ValueError, match="int32"):
        B._vector(torch.zeros(4, dtype=torch.int32), "seq_lens", torch.int32, (3,), -1)
    with pytest.raises(ValueError, match="device tensors"):
        B._vector(torch.zeros(3, dtype=torch.int32), "seq_lens", torch.int32, (3,), 0)
    with pytest.raises(ValueError, match="device tensors"):
        B._rows(x, "x", (3, 2, 64), torch.float32, 0)


# ---- places, on the host -----------------------------------------------------------------------------------

def compiled(tmp_path, source):
    src, exe = tmp_path / "places.cpp", tmp_path / "places"
    src.write_text('#include "kv_pages.h"\n#include <cassert>\n#include <cstdio>\n#include <vector>\nusing namespace moesys;\n' + source)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I" + os.path.join(ROOT, "paper_2205_10034_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    return subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout


def test_places_on_the_host(tmp_path):
    compiled(tmp_path, """int main() {
  assert(kept_length(-1, 100) == 0 && kept_length(0, 100) == 0 && kept_length(100, 100) == 100 && kept_length(2147483647, 100) == 100);
  assert(first_place(10, 0) == 0 && first_place(10, 10) == 0 && first_place(10, 3) == 7 && first_place(0, 3) == 0 && first_place(2147483647, 1) == 2147483646);
  assert(valid_page(-1, 5) == -1 && valid_page(5, 5) == -1 && valid_page(4, 5) == 4 && valid_page(0, 0) == -1 && valid_page(2147483647, 2147483647) == -1);
}""")


def test_pages_and_parts_on_the_host(tmp_path):
    """Page numbers by multiplication equal division; the parts of a batch's row of tiles hold every tile once, and every
    unfinished piece has a slot of its own where the join finds it."""
    compiled(tmp_path, """
unsigned long long seed = 1;
unsigned next() { seed = seed * 6364136223846793005ull + 1442695040888963407ull; return (unsigned)(seed >> 33); }
int main() {
  for (int d : {1, 2, 3, 5, 7, 16, 20, 100, 1000, 65535, 65536, 65537, 1000003, 1 << 30, (1 << 30) + 1, 2147483646, 2147483647}) {
    const PageDivisor q = page_divisor(d);
    for (int i = 0; i < 20000; ++i) { const int p = (int)(next() & 2147483647u); assert(q.quotient(p) == p / d); }
    for (long long k = 0; k < 50; ++k)
      for (int e = -1; e < 2; ++e) { const long long p = k * d + e; if (p >= 0 && p < 2147483648ll) assert(q.quotient((int)p) == (int)(p / d)); }
    for (int e = 0; e < 100; ++e) assert(q.quotient(2147483647 - e) == (2147483647 - e) / d);
  }
  assert(kept_tiles(0, 0, 32) == 0 && kept_tiles(1, 0, 32) == 1 && kept_tiles(32, 0, 32) == 1 && kept_tiles(33, 0, 32) == 2);
  assert(kept_tiles(33, 31, 32) == 2 && kept_tiles(33, 32, 32) == 1 && kept_tiles(2147483647, 0, 32) == 67108864);
  for (int round = 0; round < 3000; ++round) {
    const int parts = 1 + next() % (round % 2 ? 1000 : 7), least = 1 + next() % 20, S = 1 + next() % 40;
    const long long cap = 1 + next() % (round % 3 ? 200 : 3000);
    std::vector<long long> tiles(S);
    long long total = 0;
    for (long long& t : tiles) { t = row_tiles(next() % 5 ? (int)(next() % (cap + 1)) : 0); assert(t >= 1); total += t; }
    long long share = share_of_row(total, 1.0 / parts, least);
    assert(share >= least && share * parts >= total);
    const long long really = total;
    const std::vector<long long> held = tiles;
    const bool aligned = round % 3 == 1 && S < parts;
    if (aligned) {  // sequences begin parts: places of whole shares, which the parts still hold
      share = share_of_row(total, 1.0 / (parts - S), least);
      total = 0;
      for (long long& t : tiles) { const long long was = t; t = aligned_tiles(t, share); assert(t >= was && t - was < share && t % share == 0); total += t; }
      assert(total <= share * parts);
    }
    // the parts walk over the row as the kernel does; every piece but whole ones has a slot of its own, where the join looks
    std::vector<int> pieces(S, 0), first(S, -1), used(2 * parts, -1);
    long long covered = 0;
    for (int w = 0; w < parts; ++w) {
      long long x = w * share, x_end = x + share < total ? x + share : total, begin = 0;
      int b = 0;
      if (x >= total) continue;
      while (begin + tiles[b] <= x) begin += tiles[b++];
      for (int no = 0; x < x_end; ++no) {
        const long long b_end = begin + tiles[b], stop = b_end < x_end ? b_end : x_end;
        const bool whole = x == begin && b_end <= x_end;
        assert(!aligned || no == 0);
        const int slot = 2 * w + (no > 0);
        if (x == begin) {
          first[b] = slot;
          assert(part_of(b_end - 1, share) == (int)((b_end - 1) / share));
          const int expected = whole ? 1 : part_of(b_end - 1, share) - w + 1;
          pieces[b] = -expected;
        }
        if (!whole) { assert(used[slot] < 0); used[slot] = b; }
        const int j = w - first[b] / 2;
        assert(first[b] >= 0 && piece_slot(first[b], j) == slot && j < -pieces[b]);
        covered += aligned ? (b_end <= x_end ? held[b] : x_end - begin) - (x - begin) : stop - x;
        if (b_end <= x_end) assert(j == -pieces[b] - 1);
        x = b_end; begin = b_end; ++b;
      }
    }
    assert(covered == really);
  }
  for (int i = 0; i < 200000; ++i) {
    const long long share = 1 + next() % (i % 2 ? 50 : 1 << 24), part = next() % 2000;
    for (int e = -1; e < 2; ++e) if (part * share + e >= 0) assert(part_of(part * share + e, share) == (part * share + e) / share);
    // sequences of a part, as the kernel rounds them up
    const int S = 1 + next() % (i % 3 ? 600 : 1 << 30), parts = 1 + next() % (i % 5 ? 2048 : 1 << 20);
    assert(share_of_row(S, 1.0 / parts, 1) == ((long long)S + parts - 1) / parts);
  }
  // the quotient in float64, at its worst
  for (long long total : {1ll, 2ll, 3ll, 1000000007ll, (1ll << 40) - 1, 1ll << 40, (1ll << 40) + 1})
    for (int parts = 1; parts < 3000; ++parts) assert(share_of_row(total, 1.0 / parts, 1) == (total + parts - 1) / parts);
}""")
