"""Steps of drafted decoding as a server makes them: room for the drafts, their keys and values, the attention of the tree, log-probabilities, the
accepted path to its places, pages back, sequences that end and are forked; against a host that keeps every sequence's rows in a list."""
import numpy as np
import pytest
import torch

import paper_2205_10034_amd as M
from attention_util import DT, HALF_STEP
from drafts_util import tree_words
from oracle import drafts_oracle as O

pytestmark = pytest.mark.gpu

dev = lambda x, dt=np.int32: torch.from_numpy(np.ascontiguousarray(x, dtype=dt)).cuda()  # noqa: E731


def softmax_attention(q, keys, values):
    """q [heads, D] over keys, values [n, kv heads, D], in 64 bits."""
    G = q.shape[0] // keys.shape[1]
    k, v = (np.repeat(x, G, 1).astype(np.float64) for x in (keys, values))
    z = np.einsum("hd,nhd->hn", q.astype(np.float64), k) * q.shape[1] ** -0.5
    e = np.exp(z - z.max(1, keepdims=True))
    return np.einsum("hn,nhd->hd", e / e.sum(1, keepdims=True), v)


@pytest.mark.parametrize("dtype,hq,hkv,D,n,layout", [("f32", 4, 2, 64, 5, "token_major"), ("bf16", 8, 2, 64, 6, "head_major"), ("bf16", 16, 2, 128, 9, "token_major")])
def test_steps_of_drafted_decoding(dtype, hq, hkv, D, n, layout):
    S, page, width, V, K = 6, 8, 12, 301, 4
    n_pages = S * width
    rng = np.random.default_rng(n)
    shape = (n_pages, page, hkv, D) if layout == "token_major" else (n_pages, hkv, page, D)
    k, v = (torch.full(shape, float("nan"), dtype=DT[dtype], device="cuda") for _ in range(2))
    cache = M.KVCache(k, v, torch.full((S, width), -1, dtype=torch.int32, device="cuda"), layout=layout)
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    ws_pages = torch.empty(M.moe_kv_pages_workspace_bytes(cache), dtype=torch.uint8, device="cuda")
    ws_tree = torch.empty(M.moe_attention_tree_workspace_bytes(cache, hq, n), dtype=torch.uint8, device="cuda")
    ws_probs = torch.empty(M.moe_token_logprobs_workspace_bytes(S * n, V, K), dtype=torch.uint8, device="cuda")
    missing = torch.zeros(1, dtype=torch.int32, device="cuda")
    head = (torch.randn(hq * D, V, generator=torch.Generator().manual_seed(1)) * 0.3).to(DT[dtype]).cuda()
    pages = O.Pages(np.full((S, width), -1), np.zeros(n_pages), page)
    held = [[] for _ in range(S)]                      # every sequence's (key row, value row)
    lens = np.zeros(S, dtype=np.int32)
    lens[3:] = -1                                      # slots without a sequence
    d_lens = dev(lens)
    forked = 0

    for step in range(7):
        # room for the drafts, whose lengths the attention counts
        M.moe_kv_reserve(cache, refs, d_lens, ws_pages, more=n, missing=missing)
        assert pages.reserve(lens, n) == 0 and missing.item() == 0
        assert cache.page_table.cpu().tolist() == pages.table and refs.cpu().tolist() == pages.refs
        counts = [int(rng.integers(1, n + 1)) if x >= 0 else 0 for x in lens]
        first, T = np.concatenate([[0], np.cumsum(counts)]), sum(counts)
        words = tree_words(counts, seed=step)
        new = [torch.from_numpy(rng.standard_normal((T, h, D), dtype=np.float32)).to(DT[dtype]) for h in (hkv, hkv, hq)]
        seq = np.repeat(np.arange(S), counts)
        i = np.arange(T) - first[seq]
        M.moe_kv_append(cache, new[0].cuda(), new[1].cuda(), dev(lens[seq] + i), token_seq=dev(seq))
        q, total = new[2].cuda(), dev(np.maximum(lens, 0) + counts)
        out = torch.empty_like(q)
        M.moe_attention_tree(cache, q, dev(first), total, out, ws_tree, n, visible=dev(words, np.int64))

        rows = [x.float().numpy() for x in new]
        got, seen = out.float().cpu().numpy(), [[j for j in range(counts[s]) if int(words[t]) >> j & 1] for t, s in enumerate(seq)]
        for t, s in enumerate(seq):
            mine = held[s] + [(rows[0][first[s] + j], rows[1][first[s] + j]) for j in seen[t]]
            keys, values = (np.stack([m[x] for m in mine]) for x in (0, 1))
            want = softmax_attention(rows[2][t], keys, values)
            # as check_tree: D products and n weights in float32, weights of 17 bits, one rounding; scores below 16, values below 5
            size = np.abs(values).max()
            assert np.abs(got[t] - want).max() <= 2 * size * ((D + len(mine) + 300) * 2.0 ** -24 + (2.0 ** -17 if dtype == "bf16" else 0)) + HALF_STEP[dtype] * 1.01 * np.abs(want).max()

        # the verdict on the drafts
        logits = out.flatten(1) @ head
        logp, lse, ids = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), rng.integers(0, V, T)
        top_ids, top_logp = torch.empty(T, K, dtype=torch.int32, device="cuda"), torch.empty(T, K, device="cuda")
        M.moe_token_logprobs(logits, dev(ids), ws_probs, logp=logp, lse=lse, top_ids=top_ids, top_logp=top_logp)
        want_logp, _, _, order, *_ = O.logprobs(logits.float().cpu().numpy(), ids, 1.0, K)
        # (8 sqrt V + 32 roundings of the sum, and some of logits below 40 in size: 2^-24 (171 + 16 * 40))
        assert np.array_equal(top_ids.cpu().numpy(), order) and np.abs(logp.cpu().numpy() - want_logp).max() < 1e-4

        # the deepest path of the likelier half is kept, in order
        keep = np.full((S, n), -1)
        for s in range(S):
            mine = [t for t in range(T) if seq[t] == s]
            if mine:
                best = max(mine, key=lambda t: (len(seen[t]), -t))
                keep[s, :len(seen[best])] = seen[best]
                held[s] += [(rows[0][first[s] + j], rows[1][first[s] + j]) for j in seen[best]]
        base = np.maximum(lens, 0)
        new_lens = torch.empty(S, dtype=torch.int32, device="cuda")
        M.moe_kv_compact(cache, dev(base), dev(keep), new_lens=new_lens)
        now = base + (keep >= 0).sum(1)
        assert new_lens.cpu().tolist() == now.tolist()
        lens = np.where(lens >= 0, now, -1).astype(np.int32)
        if step == 4:
            lens[1], held[1] = -1, []                  # a sequence ends
        d_lens = dev(lens)
        M.moe_kv_release(cache, refs, d_lens)
        pages.release(lens)
        if step in (1, 3, 5):                          # another answer from where this one stands
            src, dst = {1: (0, 3), 3: (2, 4), 5: (3, 1)}[step]
            M.moe_kv_fork(cache, refs, dev([src]), dev([dst]), d_lens, ws_pages, missing=missing)
            as_list = lens.tolist()
            pages.fork([src], [dst], as_list)
            lens, held[dst], forked = np.array(as_list, dtype=np.int32), list(held[src]), forked + 1
        assert d_lens.cpu().tolist() == lens.tolist() and refs.cpu().tolist() == pages.refs and pages.consistent()
        assert cache.page_table.cpu().tolist() == pages.table

        # every sequence's rows lie where its table says
        pools = [(x if layout == "token_major" else x.transpose(1, 2)).float().cpu().numpy() for x in (k, v)]
        for s in range(S):
            for j, row in enumerate(held[s]):
                at = pages.table[s][j // page], j % page
                assert np.array_equal(pools[0][at], row[0]) and np.array_equal(pools[1][at], row[1]), (step, s, j)
    assert forked == 3 and max(refs.cpu().tolist()) > 1


def test_a_step_in_a_graph():
    """Attention, log-probabilities, accepted drafts and pages of one step captured together; what they read changes between the replays."""
    S, page, width, n, hq, hkv, D, V, K = 4, 16, 20, 4, 8, 2, 128, 999, 3
    g = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.randn(S * width, page, hkv, D, device="cuda", generator=g).bfloat16() for _ in range(2))
    table = torch.arange(S * width, dtype=torch.int32, device="cuda").view(S, width).contiguous()
    cache = M.KVCache(k, v, table)
    refs = torch.ones(S * width, dtype=torch.int32, device="cuda")
    q = torch.randn(S * n, hq, D, device="cuda", generator=g).bfloat16()
    head = (torch.randn(hq * D, V, device="cuda", generator=g) * 0.3).bfloat16()
    first, total, keep = dev(np.arange(S + 1) * n), dev([200, 33, 64, 100]), dev([[0, 2, -1, -1], [1, 2, 3, -1], [-1, 0, 0, 0], [0, 1, 2, 3]])
    base, new_lens, ids, missing = total - n, torch.empty(S, dtype=torch.int32, device="cuda"), dev(np.arange(S * n)), dev([0])
    out, logits = torch.empty_like(q), torch.empty(S * n, V, dtype=torch.bfloat16, device="cuda")
    logp, top_ids, top_logp = torch.empty(S * n, device="cuda"), torch.empty(S * n, K, dtype=torch.int32, device="cuda"), torch.empty(S * n, K, device="cuda")
    ws = [torch.empty(b, dtype=torch.uint8, device="cuda") for b in (M.moe_attention_tree_workspace_bytes(cache, hq, n), M.moe_token_logprobs_workspace_bytes(S * n, V, K), M.moe_kv_pages_workspace_bytes(cache))]

    def step():
        M.moe_attention_tree(cache, q, first, total, out, ws[0], n)
        torch.mm(out.flatten(1), head, out=logits)
        M.moe_token_logprobs(logits, ids, ws[1], logp=logp, top_ids=top_ids, top_logp=top_logp)
        M.moe_kv_compact(cache, base, keep, new_lens=new_lens)
        M.moe_kv_release(cache, refs, new_lens)
        M.moe_kv_reserve(cache, refs, new_lens, ws[2], more=n, missing=missing)

    state = [k, v, table, refs]
    start = [t.clone() for t in state]
    results = [out, logits, logp, top_ids, top_logp, new_lens, missing] + state

    def back(lens, seed):
        for t, s in zip(state, start):
            t.copy_(s)
        total.copy_(dev(lens))
        base.copy_(total - n)
        q.copy_(torch.randn(S * n, hq, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).bfloat16())

    step()
    torch.cuda.synchronize()
    back([200, 33, 64, 100], 3)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for lens, seed in (([200, 33, 64, 100], 3), ([4, 320, 17, 5], 4), ([50, 60, 70, 80], 5)):
        back(lens, seed)
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in results]
        back(lens, seed)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(results, want):
            assert torch.equal(a, b)
