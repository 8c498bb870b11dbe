"""Tokens decoded through one transformer block: normalisation, query/key/value projection, rotary positions and append to a
paged cache (``moe_kv_append``), attention over it (``moe_attention_decode``), output projection, and the MoE layer
(``moe_layer_forward``) - the ring workload's layer (d_model 2048, d_ff 8192, 64 experts, top-2, bf16) with 16 query heads
of 128.  The two projections and the normalisations are torch's; everything else is the library's.

    python -m paper_2205_10034_amd.block_decode_bench [--batch 1,8,64] [--context 1000,16000] [--kv-heads 4] [--steps 50]

One JSON line per batch size and context: a step's time, and what of it the cache calls and the MoE layer take.
"""
import argparse
import json
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

import torch  # noqa: E402

import paper_2205_10034_amd as M  # noqa: E402


class DecodeBlock:
    """One block with its cache for ``batch`` sequences of up to ``capacity`` tokens, pages handed out in random order."""

    def __init__(self, cfg, moe_weights, n_heads, n_kv_heads, batch, capacity, page_size=64, dtype=torch.bfloat16, seed=0):
        self.cfg, self.moe_weights, self.hq, self.hkv = cfg, moe_weights, n_heads, n_kv_heads
        d = cfg.d_model
        self.D = d // n_heads
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.w_qkv = (torch.randn(d, (n_heads + 2 * n_kv_heads) * self.D, device="cuda", generator=g) * d ** -0.5).to(dtype)
        self.w_out = (torch.randn(n_heads * self.D, d, device="cuda", generator=g) * d ** -0.5).to(dtype)
        per_seq = -(-capacity // page_size)
        table = torch.randperm(batch * per_seq, device="cuda", generator=g).to(torch.int32).view(batch, per_seq)
        pool = torch.zeros(batch * per_seq, 2, n_kv_heads, page_size, self.D, dtype=dtype, device="cuda")
        self.cache = M.KVCache(pool[:, 0], pool[:, 1], table, layout="head_major")
        self.rotary = M.Rotary(self.D, M.rotary_freqs(self.D))
        self.lens = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.places = torch.empty_like(self.lens)
        self.q_rot = torch.empty(batch, n_heads, self.D, dtype=dtype, device="cuda")
        self.attended = torch.empty_like(self.q_rot)
        self.attention_ws = torch.empty(M.moe_attention_decode_workspace_bytes(self.cache, n_heads), dtype=torch.uint8, device="cuda")
        self.moe_ws = torch.empty(M.moe_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")

    def attend(self, x):
        """x + attention of the new tokens x [batch, d_model], whose keys and values join the cache."""
        self.places.copy_(self.lens)
        self.lens.add_(1)
        qkv = (torch.nn.functional.layer_norm(x, x.shape[-1:]) @ self.w_qkv).view(-1, self.hq + 2 * self.hkv, self.D)
        q, k, v = qkv[:, :self.hq], qkv[:, self.hq:self.hq + self.hkv], qkv[:, self.hq + self.hkv:]
        M.moe_kv_append(self.cache, k, v, self.places, rotary=self.rotary, q=q, q_out=self.q_rot)
        M.moe_attention_decode(self.cache, self.q_rot, self.lens, self.attended, self.attention_ws)
        return x + self.attended.flatten(1) @ self.w_out

    def step(self, x):
        x = self.attend(x)
        y = torch.nn.functional.layer_norm(x, x.shape[-1:])
        out = torch.empty_like(x)
        M.moe_layer_forward(self.cfg, self.moe_weights, y, x, out, self.moe_ws)
        return out


def timed(f, steps):
    for _ in range(5):
        f()
    e = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
    torch.cuda.synchronize()
    e[0].record()
    for _ in range(steps):
        f()
    e[1].record()
    torch.cuda.synchronize()
    return e[0].elapsed_time(e[1]) / steps * 1e3


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--batch", default="1,8,64")
    ap.add_argument("--context", default="1000,16000")
    ap.add_argument("--kv-heads", type=int, default=4)
    ap.add_argument("--steps", type=int, default=50)
    args = ap.parse_args()
    from workloads import WORKLOADS

    base = WORKLOADS["ring"]
    E, d, f = base.E, base.d_model, base.d_ff
    g = torch.Generator(device="cuda").manual_seed(0)
    w = M.Weights({"w1": (torch.randn(E, f, d, device="cuda", generator=g) * d ** -0.5).bfloat16(),
                   "w2": (torch.randn(E, d, f, device="cuda", generator=g) * f ** -0.5).bfloat16(),
                   "w_router": (torch.randn(d, E, device="cuda", generator=g) * d ** -0.5).contiguous()})
    for batch in [int(v) for v in args.batch.split(",")]:
        for context in [int(v) for v in args.context.split(",")]:
            block = DecodeBlock(M.MoEConfig.from_workload(base.scaled(T=batch)), w, 16, args.kv_heads, batch, context + 4 * (args.steps + 5))
            block.lens.fill_(context)
            x = torch.randn(batch, d, device="cuda", generator=g).bfloat16()
            out = torch.empty_like(x)
            qkv = torch.randn(batch, 16 + 2 * args.kv_heads, block.D, device="cuda", generator=g).bfloat16()
            parts = {
                "step_us": lambda: block.step(x),
                "append_us": lambda: M.moe_kv_append(block.cache, qkv[:, 16:16 + args.kv_heads], qkv[:, 16 + args.kv_heads:], block.places,
                                                     rotary=block.rotary, q=qkv[:, :16], q_out=block.q_rot),
                "attention_us": lambda: M.moe_attention_decode(block.cache, block.q_rot, block.lens, block.attended, block.attention_ws),
                "moe_layer_us": lambda: M.moe_layer_forward(block.cfg, w, x, x, out, block.moe_ws),
            }
            print(json.dumps({"workload": f"decoded tokens through a block: batch {batch}, context {context}, 16 heads of {block.D}, {args.kv_heads} kv heads",
                              **{k: timed(v, args.steps) for k, v in parts.items()}}), flush=True)
            del block


if __name__ == "__main__":
    main()
