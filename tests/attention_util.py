"""Paged caches for the attention tests, and the bounds that the kernels' arithmetic stays within."""
import numpy as np
import torch

import paper_2205_10034_amd as M
from oracle import attention_oracle as A

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


class Paged:
    """Sequences of the given lengths over a pool in random order; every place that no sequence holds is NaN."""

    def __init__(self, lens, hkv, D, page, dtype, layout="token_major", seed=0, spare_pages=2, spare_width=1, one_pool=False, pad=0):
        g = torch.Generator().manual_seed(seed)
        self.page, self.dtype, self.hkv, self.D = page, dtype, hkv, D
        width = max([-(-n // page) for n in lens] + [0]) + spare_width
        need = sum(-(-n // page) for n in lens)
        n_pages = need + spare_pages
        order = torch.randperm(n_pages, generator=g).tolist()
        self.table = np.full((len(lens), width), -1, dtype=np.int32)
        self.k = np.full((n_pages, page, hkv, D), np.nan, dtype=np.float32)
        self.v = self.k.copy()
        for s, n in enumerate(lens):
            for i in range(-(-n // page)):
                self.table[s, i] = order.pop()
                rows = min(page, n - i * page)
                for pool in (self.k, self.v):
                    pool[self.table[s, i], :rows] = torch.randn(rows, hkv, D, generator=g).to(DT[dtype]).float().numpy()
        self.n_pages, self.layout, self.one_pool, self.pad = n_pages, layout, one_pool, pad
        self.lens = np.array(lens, dtype=np.int32)

    def cache(self, table=None):
        """The device cache: pools in the layout, each head's row padded to D + pad (strides wider than the rows), optionally
        keys and values as halves of one tensor."""
        shape = (self.n_pages, self.page, self.hkv) if self.layout == "token_major" else (self.n_pages, self.hkv, self.page)
        dt, W = DT[self.dtype], self.D + self.pad
        if self.one_pool:
            pool = torch.full((self.n_pages, 2) + shape[1:] + (W,), float("nan"), dtype=dt, device="cuda")
            kd, vd = pool[:, 0, ..., :self.D], pool[:, 1, ..., :self.D]
        else:
            kd = torch.full(shape + (W,), float("nan"), dtype=dt, device="cuda")[..., :self.D]
            vd = torch.full(shape + (W,), float("nan"), dtype=dt, device="cuda")[..., :self.D]
        for d, h in ((kd, self.k), (vd, self.v)):
            h = torch.from_numpy(h).cuda()
            d.copy_(h if self.layout == "token_major" else h.transpose(1, 2))
        t = torch.from_numpy(self.table if table is None else np.ascontiguousarray(table, dtype=np.int32)).cuda()
        return M.KVCache(kd, vd, t, layout=self.layout)

    def host(self, cache):
        """The device pools back as [pages, page_size, heads, D] float32."""
        f = lambda t: (t if self.layout == "token_major" else t.transpose(1, 2)).float().cpu().numpy()
        return f(cache.k), f(cache.v)


def queries(S, H, D, dtype, seed=1, gain=2.0):
    g = torch.Generator().manual_seed(seed)
    return (gain * torch.randn(S, H, D, generator=g)).to(DT[dtype])


def attend(cache, q, lens, **kw):
    qd = q.cuda()
    out = torch.full_like(qd, float("nan"))
    lse = torch.full(q.shape[:2], float("nan"), dtype=torch.float32, device="cuda")
    ws = torch.full((M.moe_attention_decode_workspace_bytes(cache, q.shape[1]),), 255, dtype=torch.uint8, device="cuda")
    M.moe_attention_decode(cache, qd, torch.from_numpy(np.asarray(lens, dtype=np.int32)).cuda(), out, ws, lse=lse, **kw)
    torch.cuda.synchronize()
    return out.float().cpu().numpy(), lse.cpu().numpy()


def check(p, q, lens, out, lse, table=None, scale=None, softcap=0.0, window=0, slopes=None):
    """Against the definition in 64 bits.  A score's error dz: D float32 accumulations of exact (or once rounded) products, the
    scale, cap and bias (a few roundings of |z|, the cap's tanh off by a few units in the last place of the cap).  Weights exp(z - m):
    dz, and the exponent's own rounding of |z|; bfloat16 keeps 16 bits of a weight; sums of n terms in float32.  out =
    sum w v / sum w: twice the weights' relative error, times the weighted mean of |v|, and one rounding."""
    D, dtype, e = p.D, p.dtype, 2.0 ** -24
    scale = D ** -0.5 if scale is None else scale
    ref, ref_lse, mean_abs, dot_abs, z_abs = A.decode(p.k, p.v, p.table if table is None else table, q.float().numpy(), lens, scale, softcap, window, slopes)
    n = np.maximum(np.asarray(lens), 1)[:, None]
    dz = (D + 4) * e * dot_abs + 8 * e * z_abs + 8 * e * softcap
    dw = dz + 8 * e * z_abs + (n + 16) * e + (2.0 ** -16 if dtype == "bf16" else 0.0)
    tol = 2 * dw[:, :, None] * mean_abs + HALF_STEP[dtype] * 1.01 * np.abs(ref) + 1e-37
    bad = ~(np.abs(out - ref) <= tol)
    assert not bad.any(), f"out off at {np.argwhere(bad)[:4].tolist()}: {out[bad][:4]} for {ref[bad][:4]}, allowed {tol[bad][:4]}"
    empty = np.isneginf(ref_lse)
    assert np.array_equal(np.isneginf(lse), empty), f"lse -inf at {np.argwhere(np.isneginf(lse)).tolist()}, expected {np.argwhere(empty).tolist()}"
    assert not out[empty].any()
    off = np.abs(np.where(empty, 0.0, lse) - np.where(empty, 0.0, ref_lse))
    allowed = dw + 4 * e * np.abs(np.where(empty, 0.0, ref_lse))
    assert (off <= allowed).all(), f"lse off by {off.max()}, allowed {allowed[off > allowed][:4]}"
