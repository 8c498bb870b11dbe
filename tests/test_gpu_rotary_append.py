"""Rotary positions and the append to a paged cache against the definition in 64 bits: pair layouts, axes, partial rotation, odd head
dimensions, strides and alignments, far positions, the gradient; places that are not there, and what must stay untouched."""
import numpy as np
import pytest
import torch

import paper_2205_10034_amd as M
from attention_util import DT, HALF_STEP, Paged
from oracle import attention_oracle as A

pytestmark = pytest.mark.gpu


def freqs_of(pairs):
    return np.concatenate([10000.0 ** (-np.arange(n) / max(n, 1)) for n in pairs])


def check_rotated(got, x, positions, pairs, inter, inverse, dtype):
    """Of a rotated element u c - v s: cosine and sine within 4 units of 2^-24 (angle of one turn in float32, function), three
    roundings: 8 * 2^-24 (|u| + |v|); one rounding to the type.  What passes through is equal."""
    R = 2 * sum(pairs)
    ref = A.rotary(x, positions, freqs_of(pairs), pairs, inter, inverse)
    assert np.array_equal(got[..., R:], x[..., R:])
    half = R // 2
    i = np.arange(half)
    lo, hi = (2 * i, 2 * i + 1) if inter else (i, i + half)
    size = np.zeros(x.shape[:2] + (R,))
    size[..., lo] = size[..., hi] = np.abs(x[..., lo]) + np.abs(x[..., hi])
    tol = 8 * 2.0 ** -24 * size + (HALF_STEP[dtype] * 1.01 * np.abs(ref[..., :R]) if dtype == "bf16" else 0.0)
    bad = ~(np.abs(got[..., :R] - ref[..., :R]) <= tol)
    assert not bad.any(), f"off at {np.argwhere(bad)[:4].tolist()}"


def values(T, H, D, dtype, seed=0):
    return torch.randn(T, H, D, generator=torch.Generator().manual_seed(seed)).to(DT[dtype])


def places(n_axes, T, far):
    rng = np.random.default_rng(T)
    return rng.integers(-far, far + 1, (n_axes, T)).astype(np.int32) if far else np.tile(np.arange(T, dtype=np.int32), (n_axes, 1))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("D,pairs", [(64, [32]), (128, [16, 24, 24]), (128, [32]), (80, [40]), (80, [20]), (96, [24]), (256, [40, 0, 88]), (192, [96]),
                                     (2, [1]), (7, [3]), (50, [3, 9]), (66, [33]), (34, [15])])
def test_rotary(D, pairs, inter, dtype):
    for T, H, far in ((1, 1, 0), (37, 5, 1000), (130, 3, 2_000_000_000)):
        print(T, H, D, pairs, inter, dtype, flush=True)
        x, pos = values(T, H, D, dtype), places(len(pairs), T, far)
        r = M.Rotary(D, torch.from_numpy(freqs_of(pairs)).cuda(), axis_pairs=pairs, interleaved=inter)
        xd, pd = x.cuda(), torch.from_numpy(pos).cuda()
        for inverse in (False, True):
            out = torch.full_like(xd, float("nan"))
            M.moe_rotary(r, xd, pd, out, inverse=inverse)
            check_rotated(out.float().cpu().numpy(), x.float().numpy(), pos, pairs, inter, inverse, dtype)
        inplace = xd.clone()
        M.moe_rotary(r, inplace, pd, inplace, inverse=True)
        assert torch.equal(inplace, out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rotary_strides_and_alignment(dtype):
    """Heads inside a fused projection, token-minor tensors, rows that start at odd elements: same values, nothing else written."""
    r = M.Rotary(64, M.rotary_freqs(64))
    pos = torch.arange(50, dtype=torch.int32, device="cuda")
    for token, head, first in ((20 * 64, 64, 3 * 64), (64, 50 * 64, 0), (17 * 65 + 1, 65, 3), (17 * 68, 68, 4), (17 * 66, 66, 2)):
        print(token, head, first, dtype, flush=True)
        n = first + max(49 * token + 3 * head, 0) + 64
        base = torch.randn(n, generator=torch.Generator().manual_seed(1)).to(DT[dtype]).cuda()
        x = torch.as_strided(base, (50, 4, 64), (token, head, 1), first)
        outs = torch.full((n,), 9.0, dtype=DT[dtype], device="cuda")
        out = torch.as_strided(outs, (50, 4, 64), (token, head, 1), first)
        M.moe_rotary(r, x, pos, out)
        check_rotated(out.float().cpu().numpy(), x.float().cpu().numpy(), pos.cpu().numpy()[None], [32], False, False, dtype)
        out.fill_(9.0)
        assert (outs == 9.0).all()


def test_rotary_gradient():
    """d_x of sum(d_out * rotary(x)) is the inverse rotation of d_out: against central differences of the definition, and the round
    trip returns the input."""
    pairs, T, H, D = [3, 2, 3], 5, 2, 20
    rng = np.random.default_rng(0)
    x, d_out, pos = rng.standard_normal((T, H, D)), rng.standard_normal((T, H, D)).astype(np.float32), places(3, T, 500)
    f = lambda y: float((d_out * A.rotary(y, pos, freqs_of(pairs), pairs)).sum())
    diff = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        step = np.zeros_like(x)
        step[i] = 1e-3
        diff[i] = (f(x + step) - f(x - step)) / 2e-3
    r = M.Rotary(D, torch.from_numpy(freqs_of(pairs)).cuda(), axis_pairs=pairs)
    g = torch.empty(T, H, D, device="cuda")
    pd = torch.from_numpy(pos).cuda()
    M.moe_rotary(r, torch.from_numpy(d_out).cuda(), pd, g, inverse=True)
    # linear in x: differences are off by rounding of f (sums of some 200 terms of 2^-53) over the step only
    assert np.abs(g.cpu().numpy() - diff).max() < 1e-9 + 8 * 2.0 ** -24 * 2 * np.abs(d_out).max()
    check_rotated(g.cpu().numpy(), d_out, pos, pairs, False, True, "f32")


def test_rotary_empty_and_many_heads():
    r = M.Rotary(64, M.rotary_freqs(64))
    e = torch.empty(0, 4, 64, device="cuda")
    M.moe_rotary(r, e, torch.empty(1, 0, dtype=torch.int32, device="cuda"), e)
    x, pos = values(1, 70000, 64, "bf16"), np.array([[12345]], dtype=np.int32)
    out = torch.empty_like(x, device="cuda")
    M.moe_rotary(r, x.cuda(), torch.from_numpy(pos).cuda(), out)
    check_rotated(out.float().cpu().numpy(), x.float().numpy(), pos, [32], False, False, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["token_major", "head_major"])
@pytest.mark.parametrize("D,pairs,inter,page,hq,hkv", [(64, [32], False, 16, 8, 2), (128, [16, 24, 24], False, 7, 4, 4), (128, [32], True, 1, 5, 1),
                                                      (80, [20], False, 32, 6, 3), (80, [10], True, 100, 2, 2), (8, [3], False, 3, 3, 1)])
def test_append(D, pairs, inter, page, hq, hkv, layout, dtype):
    lens = [0, 5, 33, 64]                   # places held before; the new tokens follow
    new = [3, 1, 0, 70]
    print(D, pairs, inter, page, hq, hkv, layout, dtype, flush=True)
    p = Paged([a + b for a, b in zip(lens, new)], hkv, D, page, dtype, layout, pad=8, one_pool=True)
    cache = p.cache()
    T = sum(new)
    seq = np.repeat(np.arange(4), new).astype(np.int32)
    at = np.concatenate([np.arange(a, a + b) for a, b in zip(lens, new)]).astype(np.int32)
    qkv = values(T, hq + 2 * hkv, D, dtype).cuda()
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    pos = places(len(pairs), T, 3000)
    r = M.Rotary(D, torch.from_numpy(freqs_of(pairs)).cuda(), axis_pairs=pairs, interleaved=inter)
    q_out = torch.empty(T, hq, D, dtype=DT[dtype], device="cuda")
    M.moe_kv_append(cache, k, v, torch.from_numpy(at).cuda(), token_seq=torch.from_numpy(seq).cuda(), rotary=r, positions=torch.from_numpy(pos).cuda(), q=q, q_out=q_out)
    check_rotated(q_out.float().cpu().numpy(), q.float().cpu().numpy(), pos, pairs, inter, False, dtype)
    gk, gv = p.host(cache)
    pages, rows = p.table[seq, at // page], at % page
    check_rotated(gk[pages, rows], k.float().cpu().numpy(), pos, pairs, inter, False, dtype)
    assert np.array_equal(gv[pages, rows], v.float().cpu().numpy())
    gk[pages, rows], gv[pages, rows] = p.k[pages, rows], p.v[pages, rows]
    assert np.array_equal(gk, p.k, equal_nan=True) and np.array_equal(gv, p.v, equal_nan=True)  # nothing else written


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_without_rotation_and_one_token_each(dtype):
    p = Paged([4, 9, 1], 2, 64, 4, dtype)
    cache = p.cache()
    k, v = values(3, 2, 64, dtype, 1).cuda(), values(3, 2, 64, dtype, 2).cuda()
    at = np.array([3, 8, 0], dtype=np.int32)
    M.moe_kv_append(cache, k, v, torch.from_numpy(at).cuda())
    gk, gv = p.host(cache)
    pages = p.table[np.arange(3), at // 4]
    assert np.array_equal(gk[pages, at % 4], k.float().cpu().numpy()) and np.array_equal(gv[pages, at % 4], v.float().cpu().numpy())
    # the same tokens with rotation, positions being the places
    r = M.Rotary(64, M.rotary_freqs(64))
    M.moe_kv_append(cache, k, v, torch.from_numpy(at).cuda(), rotary=r)
    gk, _ = p.host(cache)
    check_rotated(gk[pages, at % 4], k.float().cpu().numpy(), at[None], [32], False, False, dtype)


def test_append_to_places_that_are_not_there():
    p = Paged([40, 40], 1, 64, 16, "bf16", spare_pages=0, spare_width=0)
    table = p.table.copy()
    table[0, 1] = -1
    table[1, 0] = p.n_pages
    table[1, 2] = 2 ** 31 - 1
    cache = p.cache(table)
    before = [t.clone() for t in (cache.k, cache.v)]
    seq = np.array([0, 0, 1, 1, -1, 2, 0, 0, 1], dtype=np.int32)
    at = np.array([16, 31, 3, 47, 0, 0, -1, 48, 2 ** 31 - 1], dtype=np.int32)   # missing pages, sequences and places outside the table
    T = len(at)
    k = values(T, 1, 64, "bf16").cuda()
    q = values(T, 2, 64, "bf16", 3)
    q_out = torch.empty_like(q, device="cuda")
    r = M.Rotary(64, M.rotary_freqs(64))
    M.moe_kv_append(cache, k, k, torch.from_numpy(at).cuda(), token_seq=torch.from_numpy(seq).cuda(), rotary=r, q=q.cuda(), q_out=q_out)
    for was, now in zip(before, (cache.k, cache.v)):
        assert torch.equal(was.view(torch.int16), now.view(torch.int16))
    check_rotated(q_out.float().cpu().numpy(), q.float().numpy(), at[None], [32], False, False, "bf16")


def test_append_far_pages():
    """Pages beyond 2^31 elements and 2^32 bytes of a pool."""
    n_pages, page, hkv, D = 20000, 64, 16, 128
    k = torch.zeros(n_pages, page, hkv, D, dtype=torch.bfloat16, device="cuda")
    cache = M.KVCache(k, torch.zeros_like(k), torch.tensor([[19999, 5]], dtype=torch.int32, device="cuda"))
    row = values(2, hkv, D, "bf16").cuda()
    M.moe_kv_append(cache, row, row, torch.tensor([63, 64], dtype=torch.int32, device="cuda"), token_seq=torch.zeros(2, dtype=torch.int32, device="cuda"))
    for pool in (cache.k, cache.v):
        assert torch.equal(pool[19999, 63], row[0]) and torch.equal(pool[5, 0], row[1])
        assert int((pool[19999] != 0).sum()) == int((row[0] != 0).sum())


def test_append_then_attend_in_a_graph():
    """A decoded token as a serving loop runs it, captured once and replayed for the following tokens."""
    from attention_util import attend, check
    p = Paged([40, 9], 2, 64, 16, "bf16")
    cache = p.cache()
    r = M.Rotary(64, M.rotary_freqs(64))
    qkv = torch.zeros(2, 8, 64, dtype=torch.bfloat16, device="cuda")
    at, lens = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    q_rot = torch.empty(2, 4, 64, dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(q_rot)
    ws = torch.empty(M.moe_attention_decode_workspace_bytes(cache, 4), dtype=torch.uint8, device="cuda")

    def step():
        M.moe_kv_append(cache, qkv[:, 4:6], qkv[:, 6:8], at, rotary=r, q=qkv[:, :4], q_out=q_rot)
        M.moe_attention_decode(cache, q_rot, lens, out, ws)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(4):
        qkv.copy_(values(2, 8, 64, "bf16", 10 + i))
        at.copy_(torch.tensor([36 + i, 5 + i], dtype=torch.int32))
        lens.copy_(at + 1)
        g.replay()
        torch.cuda.synchronize()
        p.k, p.v = p.host(cache)
        got = out.float().cpu().numpy()
        _, lse = attend(cache, q_rot.cpu(), lens.cpu().numpy())
        check(p, q_rot.cpu(), lens.cpu().numpy(), got, lse)
