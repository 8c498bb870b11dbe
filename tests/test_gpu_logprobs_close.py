"""Log-probabilities and their gradient within bounds of each element's own rounding: every division of rows among wavefronts, in place and
not, and rows whose token is nearly certain, where 1 - p is what counts."""
import numpy as np
import pytest
import torch

import paper_2205_10034_amd as M
from attention_util import DT
from logprobs_util import Rows, confident
from test_gpu_token_logprobs import backward, forward, ids_for, logits

pytestmark = pytest.mark.gpu

# one wavefront to a row (one chunk of 1024 logits; several), four (some chunks each, or one), sixteen
SHAPES = [(1, 1), (7, 63), (300, 1000), (4099, 2050), (4096, 4001), (500, 2050), (1030, 9001), (300, 20011), (5, 17001), (1, 50001), (3, 262145), (260, 70001)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V", SHAPES)
def test_forward_and_gradient(T, V, dtype):
    rng = np.random.default_rng(V)
    x, h = logits(T, V, dtype, seed=V, stride=V + 3, offset=5)
    ids = ids_for(T, V)
    some = np.unique(np.r_[:min(T, 40), T - 1])                         # (the oracle's rows)
    rows = Rows(h[some], ids[some], 0.9)
    fwd = forward(x, ids, scale=0.9)
    rows.check_forward({k: v[some] for k, v in fwd.items()})
    g = {n: rng.standard_normal(T).astype(np.float32) for n in ("d_logp", "d_entropy", "d_lse")}
    for names in (("d_logp",), ("d_entropy",), ("d_logp", "d_entropy", "d_lse")):
        mine = {n: g[n] for n in names}
        for in_place in (False, True):
            got = backward(x.clone() if in_place else x, ids, fwd, scale=0.9, stride=V + 1, in_place=in_place, **mine)
            rows.check_gradient(got[some], dtype, **{n: v[some] for n, v in mine.items()})


@pytest.mark.parametrize("left", [0.1, 1e-2, 1e-4, 4e-6])
@pytest.mark.parametrize("T,V", [(1, 1), (9, 2), (9, 700), (4100, 1500), (40, 5000), (1, 50001), (300, 20011), (3, 140001)])
@pytest.mark.parametrize("dtype,level", [("f32", 0.0), ("f32", 20.0), ("f32", 60.0), ("f32", 100.0), ("f32", -60.0), ("bf16", 0.0), ("bf16", 20.0), ("bf16", 250.0), ("bf16", 1000.0),
                                         ("bf16", 1500.0)])
def test_confident_rows(dtype, level, T, V, left):
    """The gradient of a well predicted token is 1 - p, within its own rounding, whatever lse can say of p; with and without the entropy's."""
    some = min(T, 30)
    h, ids = confident(some, V, dtype, level, left, seed=T)
    x = torch.from_numpy(h).to(DT[dtype]).cuda().repeat(-(-T // some), 1)[:T].contiguous()
    all_ids = np.tile(ids, -(-T // some))[:T]
    rows = Rows(h, ids)
    fwd = forward(x, all_ids)
    rows.check_forward({k: v[:some] for k, v in fwd.items()})
    for ge in (None, 0.5):
        g = dict(d_logp=np.ones(T), **({} if ge is None else dict(d_entropy=np.full(T, ge))))
        for in_place in (False, True):
            got = backward(x.clone() if in_place else x, all_ids, fwd, in_place=in_place, **g)
            rows.check_gradient(got[:some], dtype, **{n: v[:some] for n, v in g.items()})


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [700, 5000, 50001])
def test_entropy_of_rows_that_another_token_dominates(V, dtype):
    """log p + entropy of the token that nearly has it all is a difference of small numbers, also where no token's own gradient is asked for."""
    h, best = confident(5, V, dtype, 30.0, 1e-3)
    ids = (best + 1) % V
    x = torch.from_numpy(h).to(DT[dtype]).cuda()
    rows, fwd = Rows(h, ids), forward(x, ids)
    for in_place in (False, True):
        for g in (dict(d_entropy=np.ones(5)), dict(d_entropy=np.ones(5), d_logp=np.full(5, -0.5))):
            rows.check_gradient(backward(x.clone() if in_place else x, ids, fwd, in_place=in_place, **g), dtype, **g)


def test_certain_rows_and_rows_of_one_logit():
    """Nothing is left for other tokens: the gradient is 0, exactly; a masked token's own is d_logp."""
    h = np.full((4, 3000), -np.inf, dtype=np.float32)
    h[0, 5], h[1, 7], h[2, 7], h[3, :2] = 60.0, -3000.0, 0.0, 1.0
    for dtype in ("bf16", "f32"):
        x = torch.from_numpy(h).to(DT[dtype]).cuda()
        fwd = forward(x, [5, 7, 9, 0])
        for in_place in (False, True):
            got = backward(x.clone() if in_place else x, [5, 7, 9, 0], fwd, in_place=in_place, d_logp=[1.0, -2.0, 3.0, 1.0])
            want = np.zeros_like(h)
            want[2, 7], want[2, 9], want[3, 0], want[3, 1] = -3.0, 3.0, 0.5, -0.5
            assert np.allclose(got, want, rtol=0, atol=2.0 ** -20) and not got[:2].any()


def test_large_batches_in_place_and_in_graphs():
    """Rows that are taken again beside rows that are not, in one captured call on changing contents."""
    T, V = 700, 9001
    x, h = logits(T, V, "bf16", gain=2.0)
    ids = ids_for(T, V)
    d_ids = torch.from_numpy(ids.astype(np.int32)).cuda()
    ws = torch.empty(M.moe_token_logprobs_workspace_bytes(T, V, 0), dtype=torch.uint8, device="cuda")
    logp, lse, ent, ones = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.ones(T, device="cuda")
    y = torch.empty_like(x)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        M.moe_token_logprobs(x, d_ids, ws, logp=logp, lse=lse, entropy=ent)
        y.copy_(x)
        M.moe_token_logprobs_backward(y, d_ids, lse, y, d_logp=ones, entropy=ent, d_entropy=ones)
    for seed in (1, 2, 3):
        h = confident(30, V, "bf16", 250.0 * seed, 1e-3, seed)[0]
        ids[:30] = h.argmax(1)
        d_ids.copy_(torch.from_numpy(ids.astype(np.int32)))
        x.copy_(logits(T, V, "bf16", seed=seed)[0])
        x[:30] = torch.from_numpy(h).to(x)
        g.replay()
        torch.cuda.synchronize()
        rows = Rows(x[:60].float().cpu().numpy(), ids[:60])
        rows.check_gradient(y[:60].float().cpu().numpy(), "bf16", d_logp=np.ones(60), d_entropy=np.ones(60))
        eager = backward(x.clone(), ids, forward(x, ids), in_place=True, d_logp=np.ones(T), d_entropy=np.ones(T))
        assert np.array_equal(eager, y.float().cpu().numpy())
