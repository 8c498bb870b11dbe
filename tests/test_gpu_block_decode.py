"""Tokens decoded through a block (append, attention, MoE layer) step by step, against the same block on the whole sequence in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2205_10034_amd as M
from paper_2205_10034_amd.block_decode_bench import DecodeBlock

pytestmark = pytest.mark.gpu


def test_decoded_tokens_equal_the_whole_sequence():
    B, d, f, E, hq, hkv, steps = 3, 256, 256, 4, 4, 2, 37
    D = d // hq
    g = torch.Generator(device="cuda").manual_seed(1)
    w = M.Weights({"w1": torch.randn(E, f, d, device="cuda", generator=g) * d ** -0.5, "w2": torch.randn(E, d, f, device="cuda", generator=g) * f ** -0.5,
                   "w_router": torch.randn(d, E, device="cuda", generator=g) * d ** -0.5})
    cfg = M.MoEConfig(T=B, d_model=d, d_ff=f, E=E, k=2, renormalize=True, dtype="f32")
    block = DecodeBlock(cfg, w, hq, hkv, B, steps + 3, page_size=8, dtype=torch.float32)
    xs = torch.randn(steps, B, d, device="cuda", generator=g)
    outs = torch.stack([block.step(x) for x in xs]).double()
    assert (block.lens == steps).all()

    # the whole sequence at once
    x = xs.double()
    norm = lambda t: torch.nn.functional.layer_norm(t, (d,))
    qkv = (norm(x) @ block.w_qkv.double()).view(steps, B, hq + 2 * hkv, D)
    angle = torch.arange(steps, device="cuda")[:, None].double() * block.rotary.freqs
    spin = torch.polar(torch.ones_like(angle), angle)[:, None, None]
    turn = lambda t: (lambda z: torch.cat([z.real, z.imag], -1))(torch.complex(t[..., :D // 2], t[..., D // 2:]) * spin)
    q, k, v = turn(qkv[:, :, :hq]), turn(qkv[:, :, hq:hq + hkv]), qkv[:, :, hq + hkv:]
    k, v = (t.repeat_interleave(hq // hkv, 2) for t in (k, v))
    z = torch.einsum("sbhd,tbhd->bhst", q, k) * D ** -0.5
    z = z.masked_fill(torch.ones(steps, steps, device="cuda").triu(1).bool(), float("-inf"))
    x = x + torch.einsum("bhst,tbhd->sbhd", torch.softmax(z, -1), v).flatten(2) @ block.w_out.double()
    y = norm(x)
    p = torch.softmax(y @ w.tensors["w_router"].double(), -1)
    top, idx = p.topk(2, -1)
    top = top / top.sum(-1, keepdim=True)
    h = torch.nn.functional.gelu(torch.einsum("sbd,efd->sbef", y, w.tensors["w1"].double()))
    e = torch.einsum("sbef,edf->sbed", h, w.tensors["w2"].double())
    want = x + (e.gather(2, idx[..., None].expand(-1, -1, -1, d)) * top[..., None]).sum(2)
    # float32 throughout: a few hundred accumulations each in two projections, the attention and two expert products, on values of size 1
    clear = (p.topk(3, -1)[0][..., 1] - p.topk(3, -1)[0][..., 2]) > 1e-4   # (a tie of the second and third expert may go either way)
    assert clear.float().mean() > 0.9
    assert float((outs - want).abs()[clear].max()) < 2e-4
