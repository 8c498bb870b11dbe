"""Log-probabilities of tokens, entropy, alternatives and their gradient against the definition in 64 bits: rows of one logit to long ones,
any alignment, ties, masked logits, rows that leave nothing, infinities and NaN."""
import numpy as np
import pytest
import torch

import paper_2205_10034_amd as M
from attention_util import DT, HALF_STEP
from oracle import drafts_oracle as O

pytestmark = pytest.mark.gpu

E = 2.0 ** -24


def logits(T, V, dtype, seed=0, gain=3.0, stride=None, offset=0):
    """Device rows `stride` elements apart, the first `offset` elements into their memory; and the values."""
    g = torch.Generator().manual_seed(seed)
    x = (gain * torch.randn(T, V, generator=g)).to(DT[dtype])
    stride = stride or V
    flat = torch.full((offset + T * stride + 8,), float("nan"), dtype=DT[dtype], device="cuda")
    view = flat[offset:offset + T * stride].as_strided((T, V), (stride, 1), offset)
    view.copy_(x)
    return view, x.float().numpy()


def forward(x, ids, K=0, scale=1.0, stream=None):
    T = x.shape[0]
    new = lambda *shape, dt=torch.float32: torch.full(shape, -99, dtype=dt, device="cuda")  # noqa: E731
    r = dict(logp=new(T), lse=new(T), entropy=new(T), top_ids=new(T, K, dt=torch.int32) if K else None, top_logp=new(T, K) if K else None)
    ws = torch.full((M.moe_token_logprobs_workspace_bytes(T, x.shape[1], K),), 255, dtype=torch.uint8, device="cuda")
    M.moe_token_logprobs(x, torch.from_numpy(np.asarray(ids, dtype=np.int32)).cuda(), ws, scale=scale, stream=stream, **r)
    torch.cuda.synchronize()
    return {k: v.cpu().numpy() for k, v in r.items() if v is not None}


def check(got, h, ids, K=0, scale=1.0):
    """A difference d = x - m is rounded once and scaled with another rounding; exp to a few units; sums of V terms in float32, in
    some tree; logarithm, and one rounding each of what is added up.  d is below |z| of the largest two."""
    V = h.shape[1]
    logp, lse, entropy, order, top_logp, p = O.logprobs(h, ids, scale, K)
    z = np.abs(np.where(np.isfinite(h), h, 0.0)).max(1) * scale
    rel = (8 * np.sqrt(V) + 32) * E + 8 * E * z          # of the sum; (errors of V roundings add up as the square root of V, eight times over)
    with np.errstate(invalid="ignore"):
        tiny = 1e-37
        for name, want, tol in (("lse", lse, rel + 4 * E * np.abs(lse)), ("logp", logp, rel + 4 * E * np.abs(logp) + 4 * E * z),
                                ("entropy", entropy, rel * (np.abs(entropy) + 2 + np.log(V)))):
            x = got[name]
            same = (np.isnan(x) & np.isnan(want)) | (x == want) | (np.abs(x - want) <= tol + tiny)
            assert same.all(), f"{name} off at {np.argwhere(~same)[:4].tolist()}: {x[~same][:4]} for {want[~same][:4]}, allowed {np.broadcast_to(tol, x.shape)[~same][:4]}"
        if K:
            assert np.array_equal(got["top_ids"], order)
            x, tol = got["top_logp"], (rel + 4 * E * z)[:, None] + 4 * E * np.abs(top_logp)
            same = (np.isnan(x) & np.isnan(top_logp)) | (x == top_logp) | (np.abs(x - top_logp) <= tol)
            assert same.all(), f"top_logp off: {x[~same][:4]} for {top_logp[~same][:4]}"


def ids_for(T, V, seed=0):
    ids = np.random.default_rng(seed).integers(0, V, T)
    if T > 3:
        ids[1], ids[2] = -1, V
    return ids


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,K", [(1, 1, 1), (3, 2, 2), (5, 7, 7), (2, 63, 5), (4, 64, 64), (7, 65, 1), (33, 1000, 20), (5, 4097, 64), (1, 50001, 5), (2, 131071, 64), (3, 262145, 3),
                                   (600, 333, 10), (2500, 40, 4), (17, 8192, 0), (64, 20011, 16), (1, 1 << 20, 8)])
def test_sizes(T, V, K, dtype):
    x, h = logits(T, V, dtype)
    ids = ids_for(T, V)
    check(forward(x, ids, K), h, ids, K)
    check(forward(x, ids, K, scale=0.37), h, ids, K, scale=0.37)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,K", [(40, 120, 20), (40, 120, 64), (33, 300, 20), (20, 500, 64), (20, 700, 63), (20, 1024, 64), (15, 1900, 64), (15, 2500, 64), (9, 8000, 64), (9, 8192, 17), (5, 9000, 64),
                                   (5, 33000, 64), (3, 70000, 33)])
def test_alternatives_of_rows_of_every_length(T, V, K, dtype):
    """One wavefront or four to a row, as many groups as alternatives and fewer, more candidates than are ranked at once."""
    for seed in range(3):
        x, h = logits(T, V, dtype, seed=seed)
        check(forward(x, [0] * T, K), h, [0] * T, K)
    x.copy_(torch.from_numpy(np.round(h)).to(DT[dtype]))          # many ties
    check(forward(x, [0] * T, K), x.float().cpu().numpy(), [0] * T, K)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("offset", [0, 1, 3, 4, 7])
def test_alignments(offset, dtype):
    for V, stride in ((1, 1), (5, 9), (131, 131), (1027, 1032), (9001, 9003), (70001, 70007)):
        x, h = logits(6, V, dtype, stride=stride, offset=offset)
        ids = ids_for(6, V)
        check(forward(x, ids, min(V, 9), scale=1.7), h, ids, min(V, 9), scale=1.7)
    x, h = logits(1, 3000, dtype, offset=offset)
    x = x.expand(4, 3000)                         # one row for all
    check(forward(x, [5, 6, 7, -1], 3), np.repeat(h, 4, 0), [5, 6, 7, -1], 3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [5, 64, 4099, 100003])
def test_ties_go_to_the_lowest_index(V, dtype):
    K = min(V, 64)
    h = np.zeros((6, V), dtype=np.float32)
    h[1, ::2] = -0.0                              # zeros are equal whatever their sign
    h[2] = np.arange(V) % 3
    h[3, V // 2:] = 1.0
    h[4] = -np.float32(1.5)
    h[5, -1] = 2.0
    x = torch.from_numpy(h).to(DT[dtype]).cuda()
    check(forward(x, [0, 1, 2, 3, 4, 0], K), h, [0, 1, 2, 3, 4, 0], K)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("order", ["rising", "falling", "stripes", "blocks"])
def test_largest_logits_lie_together(order, dtype):
    """The ways of a row that fill one thread's or one part's share with all that is largest."""
    V = 60000
    rank = np.arange(V)
    value = {"rising": rank, "falling": V - rank, "stripes": -(rank % 4096) * 20 - rank // 4096, "blocks": (rank // 8 % 512 == 3) * 1000 + rank % 8}[order]
    h = np.float32(value) / 512
    x = torch.from_numpy(np.stack([h, h[::-1], np.roll(h, 12345)]).copy()).to(DT[dtype])
    ids = [0, V - 1, 17]
    check(forward(x.cuda(), ids, 64), x.float().numpy(), ids, 64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [9, 700, 40001])
def test_masked_rows_infinities_and_nan(V, dtype):
    x, h = logits(8, V, dtype)
    lowest = np.float32(torch.finfo(DT[dtype]).min)
    h[0, ::2] = -np.inf
    h[1] = -np.inf                                # nothing is left
    h[2] = -np.inf
    h[2, V // 2] = 1.25                           # one token is left
    h[3] = lowest                                 # a mask of the type's lowest value
    h[3, 1] = 0.5
    h[4] = lowest                                 # and one that leaves nothing: all equal
    h[5, 3] = np.inf
    h[6, V - 1] = np.nan
    h[7, 4], h[7, 5], h[7, 6] = np.nan, np.inf, -np.inf
    x.copy_(torch.from_numpy(h).to(DT[dtype]))
    ids = [0, 3, V // 2, 1, 2, 3, 0, 5]
    for scale in (1.0, 0.5):
        got = forward(x, ids, 9, scale=scale)
        check(got, h, ids, 9, scale=scale)
    assert got["logp"][0] == -np.inf and got["entropy"][1] == 0 and got["entropy"][2] == 0 and got["logp"][2] == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_logits(dtype):
    for gain in (100.0, 30000.0):
        x, h = logits(9, 5000, dtype, gain=gain)
        ids = h.argmax(1)
        check(forward(x, ids, 5), h, ids, 5)
        check(forward(x, ids, 5, scale=1e-3), h, ids, 5, scale=1e-3)


def test_each_output_alone():
    x, h = logits(5, 3001, "bf16")
    ids = ids_for(5, 3001)
    all_of_them = forward(x, ids, 7)
    d_ids = torch.from_numpy(ids.astype(np.int32)).cuda()
    ws = torch.empty(M.moe_token_logprobs_workspace_bytes(5, 3001, 7), dtype=torch.uint8, device="cuda")
    for name in ("logp", "lse", "entropy"):
        out = torch.empty(5, device="cuda")
        M.moe_token_logprobs(x, d_ids if name == "logp" else None, ws, **{name: out})
        assert np.array_equal(out.cpu().numpy(), all_of_them[name])
    ti, tl = torch.empty(5, 7, dtype=torch.int32, device="cuda"), torch.empty(5, 7, device="cuda")
    M.moe_token_logprobs(x, None, ws, top_ids=ti, top_logp=tl)
    assert np.array_equal(ti.cpu().numpy(), all_of_them["top_ids"]) and np.array_equal(tl.cpu().numpy(), all_of_them["top_logp"])


def backward(x, ids, fwd, scale=1.0, in_place=False, stride=None, stream=None, **grads):
    f = lambda v: None if v is None else torch.from_numpy(np.asarray(v, dtype=np.float32)).cuda()  # noqa: E731
    T, V = x.shape
    stride = stride or V
    room = torch.full((T * stride + 8,), 7.0, dtype=x.dtype, device="cuda")
    d = x if in_place else room.as_strided((T, V), (stride, 1), 3)
    M.moe_token_logprobs_backward(x, None if ids is None else torch.from_numpy(np.asarray(ids, dtype=np.int32)).cuda(), f(fwd["lse"]), d,
                                  entropy=f(fwd["entropy"]), scale=scale, stream=stream, **{k: f(v) for k, v in grads.items()})
    torch.cuda.synchronize()
    out = d.float().cpu().numpy()
    if not in_place:
        d.fill_(7.0)
        assert (room == 7.0).all(), "written outside the gradient"
    return out


def check_gradient(got, h, ids, dtype, scale=1.0, **grads):
    """p = exp(z - lse): the roundings of z and lse (absolute, of numbers up to |z| + log V) and what lse's own sum carries; then a few
    roundings of each term, and the last one."""
    V = h.shape[1]
    want, size = O.logprobs_gradient(h, ids, scale, **grads)
    z = np.abs(np.where(np.isfinite(h), h, 0.0)).max(1) * scale + np.log(V)
    rel = (8 * np.sqrt(V) + 32) * E + 16 * E * z
    tol = 2 * rel[:, None] * (1 + np.log(V) + z[:, None]) * size + HALF_STEP[dtype] * 1.01 * np.abs(want) + 1e-37
    with np.errstate(invalid="ignore"):
        ok = (np.abs(got - want) <= tol) | (np.isnan(got) & np.isnan(want))
    assert ok.all(), f"off at {np.argwhere(~ok)[:4].tolist()}: {got[~ok][:4]} for {want[~ok][:4]}, allowed {tol[~ok][:4]}"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V", [(1, 1), (3, 2), (5, 7), (4, 64), (9, 1001), (2, 50001), (300, 333), (1, 262145)])
def test_gradient(T, V, dtype):
    rng = np.random.default_rng(T + V)
    for offset, stride in ((0, V), (3, V + 5)):
        x, h = logits(T, V, dtype, offset=offset, stride=stride)
        ids = ids_for(T, V)
        g = dict(d_logp=rng.standard_normal(T).astype(np.float32), d_entropy=rng.standard_normal(T).astype(np.float32), d_lse=rng.standard_normal(T).astype(np.float32))
        for names in (("d_logp",), ("d_entropy",), ("d_lse",), ("d_logp", "d_entropy", "d_lse")):
            mine = {n: g[n] for n in names}
            fwd = forward(x, ids, scale=1.3)
            check_gradient(backward(x, ids if "d_logp" in mine else None, fwd, scale=1.3, stride=V + offset, **mine), h, ids, dtype, scale=1.3, **mine)
        check_gradient(backward(x, ids, fwd, scale=1.3, in_place=True, **g), h, ids, dtype, scale=1.3, **g)


def test_gradient_against_differences():
    """Central differences of the forward definition, in 64 bits, over whole rows."""
    V, step = 37, 1e-5
    x, h = logits(3, V, "f32")
    ids, gs = [4, -1, 36], dict(d_logp=[1.0, 2.0, -0.5], d_entropy=[0.3, -1.0, 2.0], d_lse=[0.0, 0.7, -0.2])
    got = backward(x, ids, forward(x, ids, scale=0.8), scale=0.8, **gs)

    def value(h):
        logp, lse, entropy, *_ = O.logprobs(h, ids, 0.8)
        return np.asarray(gs["d_logp"]) * logp + np.asarray(gs["d_entropy"]) * entropy + np.asarray(gs["d_lse"]) * lse

    for j in range(V):
        up, down = np.float64(h), np.float64(h)
        up[:, j] += step
        down[:, j] -= step
        # third derivatives are of size 1: 1e-10 from the step, 1e-15 / 1e-5 from 64 bits
        assert np.abs((value(up) - value(down)) / (2 * step) - got[:, j]).max() < 1e-5


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradient_of_masked_rows(dtype):
    V = 600
    x, h = logits(7, V, dtype)
    h[0, ::2] = -np.inf
    h[1] = -np.inf
    h[2], h[2, 5] = -np.inf, 1.0
    h[3, 7] = np.nan                               # a row that no loss counts
    h[4, 7] = np.nan
    h[5, 9] = np.inf
    x.copy_(torch.from_numpy(h).to(DT[dtype]))
    ids = [1, 3, 5, -1, 2, -1, 0]
    fwd = forward(x, ids)
    g = dict(d_logp=[1.0] * 7, d_entropy=[0.5, 0.5, 0.5, 0.0, 0.0, 0.0, 0.5])
    got = backward(x, ids, fwd, **g)
    check_gradient(got, h, ids, dtype, **g)
    assert not got[1].any() and not got[3].any() and not got[5].any() and np.isnan(got[4]).all() and not got[0, ::2].any()
    # the token's own logit masked: its gradient is d_logp itself
    got = backward(x, [0] * 7, forward(x, [0] * 7), d_logp=[2.0] * 7)
    assert got[0, 0] == 2.0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [3, 700, 50001])
def test_gradient_of_logits_far_from_zero(V, dtype):
    """lse cannot hold log V beside the type's lowest value, or 2^-12 beside 2^20: rows of such logits have the gradients of the same ones near zero."""
    g = torch.Generator().manual_seed(V)
    near = torch.randint(-8, 8, (4, V), generator=g).float() / 4
    near[1] = 0.0
    for far in (float(torch.finfo(DT[dtype]).min), 2.0 ** (20 if dtype == "f32" else 8), -(2.0 ** (20 if dtype == "f32" else 8))):
        rows = near.clone() if abs(far) < 1e9 else torch.zeros(4, V)
        # (sums are exact: multiples of 1/4 below 2^21, in bfloat16 multiples of 2 from 2^8 on)
        rows = rows * (8 if dtype == "bf16" and abs(far) < 1e9 else 1)
        x0, x1 = rows.to(DT[dtype]).cuda(), (rows + far).to(DT[dtype]).cuda()
        assert torch.equal(x1.double() - far, x0.double())
        ids = [0, 1, V - 1, -1]
        g = dict(d_logp=[1.0, -2.0, 0.5, 3.0], d_entropy=[0.5, 0.5, 0.0, 1.0], d_lse=[0.0, 0.25, 0.0, -1.0])
        got = [backward(x, ids, forward(x, ids), **g) for x in (x0, x1)]
        # (in place the rows lie elsewhere, and a sum's order follows a row's alignment: the same bound, not the same bits)
        got.append(backward(x1.clone(), ids, forward(x1, ids), in_place=True, **g))
        h = x0.float().cpu().numpy()
        for d in got:
            check_gradient(d, h, ids, dtype, **g)


def test_results_do_not_change_streams_and_graphs():
    for T, V, K in ((3, 70001, 20), (700, 3001, 5)):
        x, h = logits(T, V, "bf16")
        ids = ids_for(T, V)
        first = forward(x, ids, K)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        again = forward(x, ids, K, stream=s)
        assert all(np.array_equal(first[k], again[k]) for k in first)
        d_ids = torch.from_numpy(ids.astype(np.int32)).cuda()
        ws = torch.empty(M.moe_token_logprobs_workspace_bytes(T, V, K), dtype=torch.uint8, device="cuda")
        logp, lse, ent, tl = (torch.empty(T, *n, device="cuda") for n in ((), (), (), (K,)))
        ti, d_x, ones = torch.empty(T, K, dtype=torch.int32, device="cuda"), torch.empty_like(x), torch.ones(T, device="cuda")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            M.moe_token_logprobs(x, d_ids, ws, logp=logp, lse=lse, entropy=ent, top_ids=ti, top_logp=tl)
            M.moe_token_logprobs_backward(x, d_ids, lse, d_x, d_logp=ones, entropy=ent, d_entropy=ones)
        for seed in (5, 6, 7):
            x.copy_(logits(T, V, "bf16", seed=seed)[0])
            g.replay()
            torch.cuda.synchronize()
            eager = forward(x, ids, K)
            assert np.array_equal(eager["logp"], logp.cpu().numpy()) and np.array_equal(eager["entropy"], ent.cpu().numpy())
            assert np.array_equal(eager["top_ids"], ti.cpu().numpy()) and np.array_equal(eager["top_logp"], tl.cpu().numpy())
            want = backward(x, ids, eager, d_logp=np.ones(T), d_entropy=np.ones(T))
            assert np.array_equal(want, d_x.float().cpu().numpy())


def test_rows_beyond_32_bits():
    T, V = 20000, 120001                           # 2.4e9 elements, 4.8 GB
    x = torch.zeros(T, V, dtype=torch.bfloat16, device="cuda")
    rows = [0, 17895, 17896, T - 1]
    g = torch.Generator(device="cuda").manual_seed(1)
    for r in rows:
        x[r] = torch.randn(V, device="cuda", generator=g).bfloat16()
    ids = np.full(T, 7)
    got = forward(x, ids, 2)
    h = x[rows].float().cpu().numpy()
    check({k: v[rows] for k, v in got.items()}, h, ids[rows], 2)
    d = torch.empty_like(x)
    M.moe_token_logprobs_backward(x, torch.from_numpy(ids.astype(np.int32)).cuda(), torch.from_numpy(got["lse"]).cuda(), d, d_logp=torch.ones(T, device="cuda"))
    check_gradient(d[rows].float().cpu().numpy(), h, ids[rows], "bf16", d_logp=np.ones(4))
