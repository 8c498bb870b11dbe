"""Calls of the tree attention for the tests, and the bounds that its arithmetic stays within."""
import numpy as np
import torch

import paper_2205_10034_amd as M
from attention_util import DT, HALF_STEP
from oracle import drafts_oracle as O


def tree_words(counts, seed=0, chain=False):
    """Ancestors of every token and itself, for trees that grow by a random parent among the tokens before."""
    rng = np.random.default_rng(seed)
    words = []
    for n in counts:
        mine = []
        for i in range(n):
            parent = i - 1 if chain else int(rng.integers(-1, i)) if i else -1
            mine.append((mine[parent] if parent >= 0 else 0) | 1 << i)
        words += mine
    return np.array(words, dtype=np.uint64).view(np.int64)


def firsts(counts):
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


def attend_tree(cache, q, token_first, lens, max_new, visible=None, fill=float("nan"), **kw):
    qd = q.cuda()
    out = torch.full_like(qd, fill)
    lse = torch.full(q.shape[:2], fill, dtype=torch.float32, device="cuda")
    ws = torch.full((M.moe_attention_tree_workspace_bytes(cache, q.shape[1], max_new),), 255, dtype=torch.uint8, device="cuda")
    dev = lambda x, dt: torch.from_numpy(np.ascontiguousarray(x, dtype=dt)).cuda()  # noqa: E731
    M.moe_attention_tree(cache, qd, dev(token_first, np.int32), dev(lens, np.int32), out, ws, max_new, visible=None if visible is None else dev(visible, np.int64),
                         lse=lse, **{k: dev(v, np.float32) if isinstance(v, np.ndarray) else v for k, v in kw.items()})
    torch.cuda.synchronize()
    return out.float().cpu().numpy(), lse.cpu().numpy()


def check_tree(p, q, token_first, lens, max_new, out, lse, visible=None, table=None, scale=None, softcap=0.0, window=0, sinks=0, slopes=None):
    """Against the definition in 64 bits, with the bounds of the attention of one token: a score's error dz from D float32
    accumulations, scale, cap and bias; weights exp(z - m): dz and the exponent's rounding, for bfloat16 2^-17 from their two
    numbers; sums of n terms in float32; out = sum w v / sum w: twice the weights' relative error times the weighted mean of |v|, and
    one rounding."""
    D, dtype, e = p.D, p.dtype, 2.0 ** -24
    scale = D ** -0.5 if scale is None else scale
    ref, ref_lse, mean_abs, dot_abs, z_abs, seen = O.tree(p.k, p.v, p.table if table is None else table, q.float().numpy(), token_first, lens, max_new, visible, scale,
                                                          softcap, window, sinks, slopes)
    mine = ~np.isnan(ref_lse)
    assert np.isnan(out[~mine]).all() and np.isnan(lse[~mine]).all(), "rows of no sequence were written"
    n = np.maximum(seen, 1)[:, None]
    dz = (D + 4) * e * dot_abs + 8 * e * z_abs + 8 * e * softcap
    dw = dz + 8 * e * z_abs + (n + 16) * e + (2.0 ** -17 if dtype == "bf16" else 0.0)
    tol = 2 * dw[:, :, None] * mean_abs + HALF_STEP[dtype] * 1.01 * np.abs(ref) + 1e-37
    bad = ~(np.abs(out - ref) <= tol) & mine[:, :, None]
    assert not bad.any(), f"out off at {np.argwhere(bad)[:4].tolist()}: {out[bad][:4]} for {ref[bad][:4]}, allowed {tol[bad][:4]}"
    empty = np.isneginf(ref_lse)
    assert np.array_equal(np.isneginf(lse), empty), f"lse -inf at {np.argwhere(np.isneginf(lse)).tolist()[:9]}, expected {np.argwhere(empty).tolist()[:9]}"
    assert not out[empty].any()
    off = np.abs(np.where(empty, 0.0, lse) - np.where(empty, 0.0, ref_lse))
    allowed = dw + 4 * e * np.abs(np.where(empty, 0.0, ref_lse))
    assert (off <= allowed)[mine].all(), f"lse off by {off[mine].max()}, allowed {allowed[(off > allowed) & mine][:4]}"
