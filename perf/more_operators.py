"""A step of drafted tokens over a paged cache, operator by operator: attention for a tree of drafted tokens with windows and
sinks (``moe_attention_tree``), the cache's pages and places (``moe_kv_compact``; ``moe_kv_release``, ``moe_kv_fork`` and
``moe_kv_reserve`` as one step of a server calls them), and log-probabilities of given tokens with entropy and alternatives
(``moe_token_logprobs``), with their gradient (``moe_token_logprobs_backward``).

``run`` computes a case either through the package (``own``) or in its plain form: elementary torch operations in 32 bits, one
rounding at the end.  ``exact`` is the definition in 64 bits.

Head counts and head dimensions are those of layers of the repository's workloads (d_model 1024 as 16 heads of 64, 768 as 12
of 64, 4096 as 32 of 128 with 8 key-value heads) and generic ones; vocabularies are generic.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
ES = {"bf16": 2, "f32": 4}


# ---- cases ------------------------------------------------------------------------------------------

def _case(base, name, kw):
    c = {**base, **kw}
    if name:
        c["name"] = name
    return c


def _tree(name, **kw):
    return _case(dict(op="tree", B=1, n=4, ragged=False, chain=False, hq=16, hkv=16, D=64, page=16, layout="token", dtype="bf16", lo=1, hi=128, spare=0, cap=0.0,
                      window=0, sinks=0, slopes=False, lse=False), name, kw)


def _compact(name, **kw):
    return _case(dict(op="compact", B=1, n=4, lo=1, hi=128, hkv=16, D=64, page=16, layout="token", dtype="bf16"), name, kw)


def _pages(name, **kw):
    return _case(dict(op="pages", B=1, forks=0, more=8, lo=1, hi=128, pool=0, hkv=16, D=64, page=16, layout="token", dtype="bf16"), name, kw)


def _probs(name, **kw):
    return _case(dict(op="probs", T=1, V=1000, K=0, entropy=True, scale=1.0, dtype="bf16", pad=0, masked=False), name, kw)


def _train(name, **kw):
    return _case(dict(op="train", T=1, V=1000, entropy=True, scale=1.0, dtype="bf16", pad=0, masked=False), name, kw)


def listed():
    return [
        # one request with a short prompt and five drafted tokens: the smallest call, launches and latency
        _tree("tree_one", n=5, lo=173, hi=173),
        # a serving batch in the midst of its conversations, up to 16 drafted tokens each, grouped heads, small pages
        _tree("tree_batch", B=64, n=16, ragged=True, hq=32, hkv=8, D=128, lo=100, hi=8192),
        # one very long context and the largest tree: only the length can fill the machine
        _tree("tree_long", n=64, hq=32, hkv=8, D=128, page=64, layout="head", lo=131071, hi=131071, lse=True),
        # a layer that attends to a window and to the first places, capped scores, wide heads, a chain of drafts
        _tree("tree_window", B=96, n=4, chain=True, hq=16, hkv=2, D=256, page=32, layout="head", lo=4, hi=16384, cap=50.0, window=1025, sinks=4),
        # float32 run of a model with distance biases, pages that fit no tile
        _tree("tree_f32", B=13, n=7, ragged=True, hq=12, hkv=12, D=64, page=20, lo=7, hi=2000, dtype="f32", slopes=True, lse=True),
        # one request's accepted drafts to their places
        _compact("compact_one", n=5, lo=173, hi=173),
        # a full server's accepted drafts
        _compact("compact_batch", B=256, n=16, hkv=8, D=128, page=64, layout="head", lo=100, hi=2048),
        # a full server's step of pages: trimmed and finished sequences, prompts forked for several answers, room for the next drafts
        _pages("pages_batch", B=256, forks=64, more=16, pool=12000, hkv=4, D=128, page=64, lo=100, hi=4096),
        # one sampled token: its probability, the entropy and five alternatives
        _probs("probs_one", V=50001, K=5),
        # the drafts of a serving batch judged: a tempered distribution over a large vocabulary, twenty alternatives
        _probs("probs_verify", T=576, V=128000, K=20, scale=1.25),
        # policy update over a batch of texts: log-probabilities and entropy with their gradient, rows that no vector fits
        _train("train_policy", T=8192, V=50001),
        # float32 logits of a small model, some tokens left out, forbidden tokens masked
        _train("train_f32", T=1000, V=32003, entropy=False, dtype="f32", masked=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["tree", "tree", "compact", "pages", "probs", "train"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if op in ("probs", "train"):
        V = _log(rng, 100, 262144)
        K = rng.choice([0, 1, 5, 20, 64]) if op == "probs" else 0
        T = _log(rng, 1, max(1, min(16384, int((8.0e7 if K else 4.0e8) * 2 / ES[dtype] / V))))
        kw = dict(T=T, V=V, entropy=rng.random() < 0.6, scale=rng.choice([1.0, 1.0, 0.7, 1.6]), dtype=dtype, pad=rng.choice([0, 0, 1, 64]), masked=rng.random() < 0.3)
        return _probs(None, K=min(K, V), **kw) if op == "probs" else _train(None, **kw)
    D = rng.choice([64, 64, 80, 96, 128, 128, 128, 192, 256])
    hkv = rng.choice([1, 2, 4, 5, 8, 12, 16])
    page, layout = rng.choice([1, 16, 16, 20, 32, 64, 100, 128, 256]), rng.choice(["token", "head"])
    kw = dict(hkv=hkv, D=D, page=page, layout=layout, dtype=dtype)
    if op == "compact":
        n = _log(rng, 1, 64)
        hi = _log(rng, n, 4000)
        return _compact(None, B=_log(rng, 1, max(1, min(512, int(1.0e9 / (4 * hi * hkv * D * ES[dtype]))))), n=n, lo=rng.choice([n, hi]), hi=hi, **kw)
    if op == "pages":
        hi = _log(rng, 1, 8192)
        B = _log(rng, 2, max(2, min(512, int(2.0e9 / (4 * (hi + 2 * page) * hkv * D * ES[dtype])))))
        return _pages(None, B=B, forks=_log(rng, 1, max(1, B // 3)), more=rng.choice([1, 4, 16, 64]), lo=rng.choice([1, hi]), hi=hi, **kw)
    hq = hkv * rng.choice([1, 1, 2, 3, 4, 6, 8, 16])
    n = _log(rng, 1, 64)
    hi = _log(rng, n, 131072)
    # half of the largest listed case's keys and values, and of its products, at most
    limit = min(1.0e9 / (4.0 * hkv * D * ES[dtype] * hi), 0.7e11 / (4.0 * hi * n * hq * D) / (4 if dtype == "f32" else 1))
    B = min(_log(rng, 1, 512), max(1, int(limit)))
    hi = max(n, min(hi, int(hi * max(limit, 0.01)))) if limit < 1 else hi
    return _tree(None, B=B, n=n, ragged=rng.random() < 0.5, chain=rng.random() < 0.3, hq=hq, lo=rng.choice([hi, max(n, hi // 2), 1]), hi=hi, spare=rng.choice([0, 0, 3, 300]),
                 cap=rng.choice([0.0, 0.0, 30.0]), slopes=rng.random() < 0.25, lse=rng.random() < 0.4, window=rng.choice([0, 0, 0, 1, 100, 1000, 4096]),
                 sinks=rng.choice([0, 0, 4, 33]), **kw)


# ---- inputs -----------------------------------------------------------------------------------------

def _host(c):
    return random.Random(c["B"] * 1000003 + c["hi"] * 17 + c["lo"] + 31 * c["page"])


def _drafts(c):
    """New tokens of every sequence, and which of its sequence's drafts each token sees, itself among them (bits)."""
    r = _host(c)
    counts = [c["n"]] + [r.randint(1, c["n"]) if c["ragged"] else c["n"] for _ in range(c["B"] - 1)]
    bits = []
    for n in counts:
        mine = []
        for i in range(n):
            parent = i - 1 if c["chain"] else r.randint(max(-1, i - 6), i - 1)
            mine.append((mine[parent] if parent >= 0 else 0) | 1 << i)
        bits += mine
    return counts, bits


def _lens(c, least=None):
    """Lengths of the sequences with their drafts: the first has the longest, the others are spread over lo..hi."""
    r = _host(c)
    least = least or [1] * c["B"]
    return [max(least[0], c["hi"])] + [max(m, r.randint(c["lo"], c["hi"])) for m in least[1:]]


def _gen(seed, salt):
    return torch.Generator(device="cuda").manual_seed(seed * 7 + salt)


def _table(widths, width, n_pages, seed):
    """Page table [sequences, width] over a pool in random order; entries past a sequence's own are -1."""
    order = torch.randperm(n_pages, device="cuda", generator=_gen(seed, 1)).to(torch.int32)
    first = torch.tensor([0] + widths[:-1]).cumsum(0).cuda()[:, None]
    at = torch.arange(width, device="cuda")[None, :]
    return torch.where(at < torch.tensor(widths).cuda()[:, None], order[(first + at).clamp(max=n_pages - 1)], -1).to(torch.int32).contiguous()


def _pool(c, n_pages, seed, salt):
    mid = (c["page"], c["hkv"]) if c["layout"] == "token" else (c["hkv"], c["page"])
    return torch.empty((n_pages,) + mid + (c["D"],), dtype=DT[c["dtype"]], device="cuda").normal_(generator=_gen(seed, salt))


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _inputs_tree(c, seed):
    counts, bits = _drafts(c)
    lens = _lens(c, counts)
    widths = [-(-x // c["page"]) for x in lens]
    n_pages = sum(widths) + 3
    s = {"counts": counts, "host_lens": lens, "table": _table(widths, max(widths) + c["spare"], n_pages, seed), "k": _pool(c, n_pages, seed, 2), "v": _pool(c, n_pages, seed, 3)}
    s["q"] = (2.0 * torch.randn(len(bits), c["hq"], c["D"], device="cuda", generator=_gen(seed, 4))).to(DT[c["dtype"]])
    s["lens"], s["first"] = _int32(lens), torch.tensor([0] + counts).cumsum(0).to(torch.int32).cuda()
    s["visible"] = torch.tensor([b - (1 << 64) if b >> 63 else b for b in bits], dtype=torch.int64, device="cuda")
    if c["slopes"]:
        s["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / c["hq"]) for h in range(c["hq"])], dtype=torch.float32, device="cuda")
    return s


def _inputs_compact(c, seed):
    lens = _lens(c, [c["n"]] * c["B"])
    widths = [-(-x // c["page"]) for x in lens]
    n_pages = sum(widths) + 3
    s = {"table": _table(widths, max(widths), n_pages, seed), "k": _pool(c, n_pages, seed, 2), "v": _pool(c, n_pages, seed, 3)}
    s["base"] = _int32([x - c["n"] for x in lens])
    # the accepted drafts of each sequence, in order, then -1
    g = _gen(seed, 5)
    taken = torch.rand(c["B"], c["n"], device="cuda", generator=g) < torch.rand(c["B"], 1, device="cuda", generator=g)
    i = torch.arange(c["n"], device="cuda")
    order = torch.where(taken, i, i + c["n"]).sort(1)[0]
    s["keep"] = torch.where(order < c["n"], order, -1).to(torch.int32).contiguous()
    return s


def _inputs_pages(c, seed):
    """Slots of a server: each of the first `forks` is to be forked into a slot at the end, where a finished sequence still has
    pages; of the others some have finished and all have pages for drafts that were not accepted."""
    B, F, P = c["B"], c["forks"], c["page"]
    lens = _lens(c)
    held = [-(-(x + 2 * P) // P) for x in lens]
    width = max(-(-(x + c["more"]) // P) for x in lens + [c["hi"] + 2 * P])
    n_pages = max(c["pool"], sum(held) + B + 8)
    s = {"table": _table(held, width, n_pages, seed), "k": _pool(c, n_pages, seed, 2), "v": _pool(c, n_pages, seed, 3)}
    flat = s["table"][s["table"] >= 0].long()
    s["refs"] = torch.zeros(n_pages, dtype=torch.int32, device="cuda").index_add_(0, flat, torch.ones_like(flat, dtype=torch.int32))
    s["lens"] = _int32([-1 if b >= B - F or (b >= F and b % 5 == 4) else x for b, x in enumerate(lens)])
    s["src"], s["dst"] = _int32(list(range(F))), _int32([B - 1 - i for i in range(F)])
    s["missing"] = torch.zeros(2, dtype=torch.int32, device="cuda")
    return s


def _inputs_probs(c, seed):
    """Logits of a few likely tokens above a noise of others; rows are `pad` elements further apart than they are long."""
    T, V = c["T"], c["V"]
    g = _gen(seed, 6)
    x = torch.empty(T, V + c["pad"], dtype=DT[c["dtype"]], device="cuda")
    for t0 in range(0, T, 1024):
        z = torch.randn(min(1024, T - t0), V, device="cuda", generator=g)
        x[t0:t0 + 1024, :V] = 1.5 * z + 0.1 * z ** 3
    x = x[:, :V]
    if c["masked"]:
        x[:, torch.randperm(V, device="cuda", generator=g)[:V // 3]] = float("-inf")
        x[:, 0] = 1.0
    ids = torch.randint(0, V, (T,), device="cuda", generator=g)
    best = x.argmax(1)
    ids = torch.where((torch.rand(T, device="cuda", generator=g) < 0.6) | torch.isinf(x.gather(1, ids[:, None])[:, 0]), best, ids)
    if c["masked"] and T > 8:
        ids[torch.randint(0, T, (T // 8,), device="cuda", generator=g)] = -1  # prompt tokens, which no loss counts
    s = {"x": x, "ids": ids.to(torch.int32)}
    if c["op"] == "train":
        s["d_logp"] = torch.randn(T, device="cuda", generator=g) / T
        s["d_entropy"] = torch.randn(T, device="cuda", generator=g) / T if c["entropy"] else None
    return s


def _inputs(c, seed):
    s = {"tree": _inputs_tree, "compact": _inputs_compact, "pages": _inputs_pages, "probs": _inputs_probs, "train": _inputs_probs}[c["op"]](c, seed)
    s["case"] = c
    return s


def prepare(case, seed):
    c = case
    s = _inputs(c, seed)
    if c["op"] == "tree":
        s["out"] = torch.empty_like(s["q"])
        s["out_lse"] = torch.empty(s["q"].shape[:2], dtype=torch.float32, device="cuda") if c["lse"] else None
    elif c["op"] == "compact":
        s["new_lens"] = torch.empty_like(s["base"])
    elif c["op"] in ("probs", "train"):
        for name in ("logp", "lse", "entropy"):
            s[name] = torch.empty(c["T"], dtype=torch.float32, device="cuda") if name != "entropy" or c["entropy"] else None
        if c["op"] == "train":
            s["d_x"] = torch.empty_strided(s["x"].shape, s["x"].stride(), dtype=s["x"].dtype, device="cuda")
        else:
            s["top_ids"] = torch.empty(c["T"], c["K"], dtype=torch.int32, device="cuda") if c["K"] else None
            s["top_logp"] = torch.empty(c["T"], c["K"], dtype=torch.float32, device="cuda") if c["K"] else None
    if own:
        import paper_2205_10034_amd as M
        if c["op"] in ("probs", "train"):
            need = M.moe_token_logprobs_workspace_bytes(c["T"], c["V"], c.get("K", 0))
        else:
            s["cache"] = M.KVCache(s["k"], s["v"], s["table"], layout=c["layout"] + "_major")
            need = M.moe_attention_tree_workspace_bytes(s["cache"], c["hq"], c["n"]) if c["op"] == "tree" else M.moe_kv_pages_workspace_bytes(s["cache"]) if c["op"] == "pages" else 0
        s["ws"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    return s


# ---- the operators ----------------------------------------------------------------------------------

def run(state):
    c = state["case"]
    if own:
        return _run_own(c, state)
    return {"tree": _plain_tree, "compact": _plain_compact, "pages": _plain_pages, "probs": _plain_probs, "train": _plain_train}[c["op"]](c, state)


def _answer(c, s):
    if c["op"] == "tree":
        return [s["out"], s["out_lse"]] if c["lse"] else [s["out"]]
    if c["op"] == "compact":
        return [s["k"], s["v"], s["new_lens"]]
    if c["op"] == "pages":
        return [s["table"], s["refs"], s["lens"], s["missing"], s["k"], s["v"]]
    names = ["logp", "lse"] + (["entropy"] if c["entropy"] else [])
    return [s[n] for n in names + (["d_x"] if c["op"] == "train" else ["top_ids", "top_logp"] if c["K"] else [])]


def _run_own(c, s):
    import paper_2205_10034_amd as M
    if c["op"] == "tree":
        M.moe_attention_tree(s["cache"], s["q"], s["first"], s["lens"], s["out"], s["ws"], max_new=c["n"], visible=None if c["chain"] else s["visible"],
                             softcap=c["cap"], window=c["window"], sinks=c["sinks"], slopes=s.get("slopes"), lse=s["out_lse"])
    elif c["op"] == "compact":
        M.moe_kv_compact(s["cache"], s["base"], s["keep"], new_lens=s["new_lens"])
    elif c["op"] == "pages":
        M.moe_kv_release(s["cache"], s["refs"], s["lens"])
        M.moe_kv_fork(s["cache"], s["refs"], s["src"], s["dst"], s["lens"], s["ws"], missing=s["missing"][:1])
        M.moe_kv_reserve(s["cache"], s["refs"], s["lens"], s["ws"], more=c["more"], missing=s["missing"][1:])
    else:
        M.moe_token_logprobs(s["x"], s["ids"], s["ws"], logp=s["logp"], lse=s["lse"], entropy=s["entropy"], top_ids=s.get("top_ids"), top_logp=s.get("top_logp"), scale=c["scale"])
        if c["op"] == "train":
            M.moe_token_logprobs_backward(s["x"], s["ids"], s["lse"], s["d_x"], d_logp=s["d_logp"], entropy=s["entropy"], d_entropy=s["d_entropy"], scale=c["scale"])
    return _answer(c, s)


def _groups(c, s, budget):
    """Runs of sequences whose keys and scores, padded to the longest, stay below budget elements; and how many places that is."""
    per, most = c["hkv"] * max(c["D"], c["n"] * c["hq"] // c["hkv"]), c["window"] + c["n"] if c["window"] else 1 << 40
    lens = s["host_lens"]
    first = 0
    while first < len(lens):
        n, places = 0, 1
        while first + n < len(lens):
            more = max(places, min(most, lens[first + n]))
            if n and (n + 1) * more * per > budget:
                break
            n, places = n + 1, more
        yield first, first + n, places
        first += n


def _plain_tree(c, s):
    G, D, P, N = c["hq"] // c["hkv"], c["D"], c["page"], c["n"]
    for b0, b1, places in _groups(c, s, 1 << 28):
        B = b1 - b0
        n_new = (s["first"][b0 + 1:b1 + 1] - s["first"][b0:b1])[:, None]
        n = s["lens"][b0:b1, None]
        base = n - n_new
        i = torch.arange(N, device="cuda")[None, :]
        token = (s["first"][b0:b1, None] + i).clamp(max=s["q"].shape[0] - 1).long()
        bits = s["visible"][token]
        shift = torch.arange(N, device="cuda")
        sees = (bits[:, :, None] >> shift & 1).bool()                                # [B, N, N]
        depth = sees.sum(-1) - 1
        # places: all, or the sinks and what a window can reach
        if c["window"]:
            start = (n - c["window"] - N).clamp(min=0)
            first = torch.arange(c["sinks"], device="cuda")[None, :].expand(B, -1)
            rest = start + torch.arange(places + N, device="cuda")[None, :]
            at = torch.cat([torch.where(first < start, first, -1), rest], 1)
        else:
            at = torch.arange(places, device="cuda")[None, :].expand(B, -1)
        there = (at >= 0) & (at < n)
        place = torch.where(there, at, 0).long()
        draft = (place - base).clamp(0, N - 1)
        is_draft = place >= base
        pos_key = torch.where(is_draft, base + torch.gather(depth, 1, draft), place)  # [B, L]
        pos = base + depth                                                           # [B, N]
        away = pos[:, :, None] - pos_key[:, None, :]
        keep = there[:, None, :] & (~is_draft[:, None, :] | torch.gather(sees, 2, draft[:, None, :].expand(-1, N, -1)))
        if c["window"]:
            keep = keep & ((away < c["window"]) | (place < c["sinks"])[:, None, :])
        page = torch.gather(s["table"][b0:b1].long(), 1, torch.div(place, P, rounding_mode="floor"))

        def rows(pool):
            x = pool[page, place % P] if c["layout"] == "token" else pool[page, :, place % P]
            return x.float().transpose(1, 2)                                         # [B, hkv, L, D]

        q = s["q"][token].float().view(B, N, c["hkv"], G, D).permute(0, 2, 1, 3, 4).reshape(B, c["hkv"], N * G, D)
        z = torch.matmul(q, rows(s["k"]).transpose(2, 3)) * (D ** -0.5)
        if c["cap"]:
            z = torch.tanh(z / c["cap"]) * c["cap"]
        z = z.view(B, c["hkv"], N, G, -1)
        if c["slopes"]:
            z = z - s["slopes"].view(1, c["hkv"], 1, G, 1) * away[:, None, :, None, :].float()
        z = torch.where(keep[:, None, :, None, :], z, float("-inf"))
        top = z.amax(-1, keepdim=True)
        p = torch.exp(z - torch.where(top == float("-inf"), 0.0, top))
        total = p.sum(-1, keepdim=True)
        o = torch.matmul(p.flatten(2, 3), rows(s["v"])).view(B, c["hkv"], N, G, D) / torch.where(total > 0, total, 1.0)
        mine = (i < n_new)
        s["out"][token[mine]] = o.permute(0, 2, 1, 3, 4).reshape(B, N, c["hq"], D)[mine].to(s["out"].dtype)
        if c["lse"]:
            s["out_lse"][token[mine]] = (torch.log(total) + top).permute(0, 2, 1, 3, 4).reshape(B, N, c["hq"])[mine]
    return _answer(c, s)


def _plain_compact(c, s):
    n = torch.cumprod((s["keep"] >= 0).int(), 1)
    s["new_lens"].copy_(s["base"] + n.sum(1))
    seq, i = torch.nonzero(n, as_tuple=True)
    src = (s["base"][seq] + s["keep"][seq, i]).long()
    dst = (s["base"][seq] + i).long()
    P = c["page"]
    a, b = (s["table"][seq, torch.div(p, P, rounding_mode="floor")].long() for p in (src, dst))
    for pool in (s["k"], s["v"]):
        if c["layout"] == "token":
            pool[b, dst % P] = pool[a, src % P]
        else:
            pool[b, :, dst % P] = pool[a, :, src % P]
    return _answer(c, s)


def _there(c, s, entries):
    return (entries >= 0) & (entries < s["refs"].shape[0])


def _count(s, entries, there, by):
    s["refs"].index_add_(0, torch.where(there, entries, 0).flatten().long(), torch.where(there, by, 0).to(torch.int32).flatten())


def _take(s, wanted, missing):
    """The lowest free pages for the places of a matrix that want one, in order; -1 where none is left."""
    used = s["refs"] != 0
    order = torch.argsort(used, stable=True)
    rank = torch.cumsum(wanted.flatten().long(), 0).view(wanted.shape) - 1
    had = wanted & (rank < (~used).sum())
    page = torch.where(had, order[rank.clamp(0, order.shape[0] - 1)].to(torch.int32), -1)
    missing.copy_((wanted & ~had).sum())
    _count(s, page, had, 1)
    return page


def _plain_pages(c, s):
    P, table = c["page"], s["table"]
    column = torch.arange(table.shape[1], device="cuda")[None, :]
    # release
    drop = column >= torch.div(s["lens"].clamp(min=0) + P - 1, P, rounding_mode="floor")[:, None]
    _count(s, table, drop & _there(c, s, table), -1)
    table.masked_fill_(drop, -1)
    # fork
    src, dst = s["src"].long(), s["dst"].long()
    n = s["lens"][src].clamp(min=0)
    old, theirs = table[dst], table[src]
    full, part = torch.div(n, P, rounding_mode="floor"), n % P
    _count(s, old, _there(c, s, old), -1)
    new = torch.where(column < full[:, None], theirs, -1)
    _count(s, new, _there(c, s, new), 1)
    begun = theirs.gather(1, full[:, None].long().clamp(max=table.shape[1] - 1))
    page = _take(s, (part > 0)[:, None] & _there(c, s, begun), s["missing"][:1])
    table[dst] = torch.where(column == full[:, None], page, new)
    s["lens"][dst] = s["lens"][src]
    had = page[:, 0] >= 0
    a, b = begun[:, 0][had].long(), page[:, 0][had].long()
    row = torch.arange(P, device="cuda")[None, :] < part[had][:, None]
    row = row[:, :, None, None] if c["layout"] == "token" else row[:, None, :, None]
    for pool in (s["k"], s["v"]):
        pool[b] = torch.where(row, pool[a], pool[b])
    # reserve
    want = (column < torch.div(s["lens"] + c["more"] + P - 1, P, rounding_mode="floor")[:, None]) & (s["lens"] >= 0)[:, None] & ~_there(c, s, table)
    table.copy_(torch.where(want, _take(s, want, s["missing"][1:]), table))
    return _answer(c, s)


def _statistics(c, s):
    """Log-probabilities, probabilities and the three numbers of every row in 32 bits."""
    z = s["x"].float() * c["scale"]
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    s["lse"].copy_((torch.log(total) + top)[:, 0])
    has = s["ids"] >= 0
    logp = (z - top) - torch.log(total)
    s["logp"].copy_(torch.where(has, logp.gather(1, s["ids"].clamp(min=0)[:, None].long())[:, 0], 0.0))
    if c["entropy"]:
        s["entropy"].copy_(torch.log(total)[:, 0] - torch.where(e > 0, e * (z - top), 0.0).sum(1) / total[:, 0])
    return logp, e / total, has


def _plain_probs(c, s):
    logp, _, _ = _statistics(c, s)
    if c["K"]:
        # one whole number per logit that orders them by value and then by place: no ties are left to topk
        bits = (s["x"].float() + 0.0).view(torch.int32).long()
        key = torch.where(bits < 0, -(bits & 0x7fffffff) - 1, bits) * (1 << 20) + (c["V"] - torch.arange(c["V"], device="cuda"))
        ids = key.topk(c["K"], 1)[1]
        s["top_ids"].copy_(ids)
        s["top_logp"].copy_(logp.gather(1, ids))
    return _answer(c, s)


def _plain_train(c, s):
    logp, p, has = _statistics(c, s)
    g = torch.where(has, s["d_logp"], 0.0)[:, None]
    d = -g * p
    d.scatter_add_(1, s["ids"].clamp(min=0)[:, None].long(), g)
    if c["entropy"]:
        d = d - torch.where(p > 0, s["d_entropy"][:, None] * p * (logp + s["entropy"][:, None]), 0.0)
    s["d_x"].copy_(d * c["scale"])
    return _answer(c, s)


# ---- what a pass cannot do without --------------------------------------------------------------------

def work(case):
    c = case
    es = ES[c["dtype"]]
    if c["op"] in ("probs", "train"):
        size = c["T"] * c["V"]
        per_row = 4 * c["T"] * (4 + 2 * c.get("K", 0))
        # forward and backward each read the logits, and the gradient is as large
        return {"bytes": size * es * (3 if c["op"] == "train" else 1) + per_row, "flops": size * (12 if c["op"] == "train" else 5)}
    row = c["hkv"] * c["D"] * es
    if c["op"] == "tree":
        counts, bits = _drafts(c)
        lens = _lens(c, counts)
        W = c["window"] or 1 << 40
        keys = pairs = t = 0
        for n, m in zip(lens, counts):
            base = n - m
            keys += min(n, W - 1 + m + c["sinks"])
            for b in bits[t:t + m]:
                d = bin(b).count("1")
                # (cached places that the window reaches from a token d - 1 behind the cache, the sinks before them, and the drafts)
                inside = max(0, min(base, W - d))
                pairs += inside + min(c["sinks"] if c["window"] else 0, base - inside) + min(d, W)
            t += m
        return {"bytes": 2 * keys * row + 2 * t * c["hq"] * c["D"] * es + 8 * t + (4 * t * c["hq"] if c["lse"] else 0), "flops": 4 * pairs * c["hq"] * c["D"]}
    if c["op"] == "compact":
        return {"bytes": 2 * 2 * c["B"] * (c["n"] / 2) * row + 4 * c["B"] * (c["n"] + 2), "flops": 0}
    lens = _lens(c)
    held = sum(-(-(x + 2 * c["page"]) // c["page"]) for x in lens)
    copied = sum(x % c["page"] for x in lens[:c["forks"]])
    return {"bytes": 4 * max(c["pool"], held) + 8 * held + 2 * 2 * copied * row, "flops": 0}


# ---- the definition in 64 bits ------------------------------------------------------------------------

def _exact_tree(c, s):
    G, D, W = c["hq"] // c["hkv"], c["D"], c["window"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], float("-inf"), dtype=torch.float64, device="cuda")
    _, bits = _drafts(c)
    t = 0
    for b, (n, m) in enumerate(zip(s["host_lens"], s["counts"])):
        base = n - m
        depth = torch.tensor([bin(x).count("1") - 1 for x in bits[t:t + m]], device="cuda")
        j = torch.arange(n, device="cuda")
        if W:
            j = j[(j < c["sinks"]) | (j > base - W)]
        pos_key = torch.where(j < base, j, base + depth[(j - base).clamp(0, m - 1)])
        away = (base + depth)[:, None] - pos_key[None, :]
        allowed = torch.tensor([[x >> i & 1 for i in range(m)] for x in bits[t:t + m]], device="cuda").bool()
        keep = (j < base)[None, :] | allowed[:, (j - base).clamp(0, m - 1)]
        if W:
            keep &= (away < W) | (j < c["sinks"])[None, :]
        page, row = s["table"][b][torch.div(j, c["page"], rounding_mode="floor")].long(), j % c["page"]
        for h in range(c["hkv"]):
            k, v = (s["k"][page, row, h], s["v"][page, row, h]) if c["layout"] == "token" else (s["k"][page, h, row], s["v"][page, h, row])
            q = s["q"][t:t + m, h * G:(h + 1) * G].double()
            z = (q.reshape(m * G, D) @ k.double().t()).view(m, G, -1) / math.sqrt(D)
            if c["cap"]:
                z = c["cap"] * torch.tanh(z / c["cap"])
            if c["slopes"]:
                z = z - away[:, None, :].double() * s["slopes"][h * G:(h + 1) * G].double()[None, :, None]
            z = z.masked_fill(~keep[:, None, :], float("-inf"))
            lse[t:t + m, h * G:(h + 1) * G] = torch.logsumexp(z, -1)
            out[t:t + m, h * G:(h + 1) * G] = (torch.softmax(z, -1).view(m * G, -1) @ v.double()).view(m, G, D)
        t += m
    return [out, lse] if c["lse"] else [out]


def _exact_compact(c, s):
    pools = []
    for pool in (s["k"], s["v"]):
        old = pool.float()
        new = old.clone()
        a, b = (x if c["layout"] == "token" else x.transpose(1, 2) for x in (old, new))
        for seq, (base, keep) in enumerate(zip(s["base"].tolist(), s["keep"].tolist())):
            keep = [x for x in keep if x >= 0]
            src, dst = (torch.tensor([base + x for x in y], dtype=torch.int64, device="cuda") for y in (keep, range(len(keep))))
            b[s["table"][seq][dst // c["page"]].long(), dst % c["page"]] = a[s["table"][seq][src // c["page"]].long(), src % c["page"]]
        pools.append(new)
    return pools + [None]


def _exact_pages(c, s):
    """Sequence by sequence on the host."""
    P, n_pages = c["page"], s["refs"].shape[0]
    table, refs, lens = s["table"].tolist(), s["refs"].tolist(), s["lens"].tolist()
    pages = lambda n: -(-max(n, 0) // P)  # noqa: E731

    def drop(seq, first):
        for i in range(first, len(table[seq])):
            if table[seq][i] >= 0:
                refs[table[seq][i]] -= 1
            table[seq][i] = -1

    def take():
        page = next((p for p in range(n_pages) if refs[p] == 0), -1)
        if page >= 0:
            refs[page] = 1
        return page

    for seq, n in enumerate(lens):
        drop(seq, pages(n))
    forks = list(zip(s["src"].tolist(), s["dst"].tolist()))
    for a, b in forks:
        drop(b, 0)
        for i in range(lens[a] // P):
            table[b][i] = table[a][i]
            refs[table[a][i]] += 1
        lens[b] = lens[a]
    copies = []
    for a, b in forks:
        if lens[a] % P:
            table[b][lens[a] // P] = take()
            copies.append((table[a][lens[a] // P], table[b][lens[a] // P], lens[a] % P))
    pools = []
    for pool in (s["k"], s["v"]):
        new = pool.clone()
        x = new if c["layout"] == "token" else new.transpose(1, 2)
        for a, b, n in copies:
            x[b, :n] = x[a, :n]
        pools.append(new)
    return [None, None, None, None] + pools


def _exact_probs(c, s):
    logp, lse, entropy, d_x, top = [], [], [], [], []
    step = max(1, (1 << 26) // c["V"])
    for t0 in range(0, c["T"], step):
        at = slice(t0, t0 + step)
        z = s["x"][at].double() * c["scale"]
        lp = torch.log_softmax(z, 1)
        p = lp.exp()
        ids = s["ids"][at].long()
        has = ids >= 0
        h = -(p * lp.masked_fill(p == 0, 0.0)).sum(1)
        logp.append(torch.where(has, lp.gather(1, ids.clamp(min=0)[:, None])[:, 0], 0.0))
        lse.append(torch.logsumexp(z, 1))
        entropy.append(h)
        if c["op"] == "train":
            hot = torch.zeros_like(p).scatter_(1, ids.clamp(min=0)[:, None], 1.0)
            d = torch.where(has, s["d_logp"][at].double(), 0.0)[:, None] * (hot - p)
            if c["entropy"]:
                d = d - s["d_entropy"][at].double()[:, None] * p * (lp.masked_fill(p == 0, 0.0) + h[:, None])
            d_x.append((c["scale"] * d).float())  # (64 bits of the largest would not fit beside the others)
        elif c["K"]:
            top.append(lp.topk(c["K"], 1)[0])
    got = [torch.cat(logp), torch.cat(lse)] + ([torch.cat(entropy)] if c["entropy"] else [])
    return got + ([torch.cat(d_x)] if c["op"] == "train" else [None, torch.cat(top)] if c["K"] else [])


def exact(case, seed):
    s = _inputs(case, seed)
    return {"tree": _exact_tree, "compact": _exact_compact, "pages": _exact_pages, "probs": _exact_probs, "train": _exact_probs}[case["op"]](case, s)
