"""The attention half of a decoded token, operator by operator: rotary positions (``moe_rotary``), keys and values into a
paged cache (``moe_kv_append``), and attention of one new token per sequence over that cache (``moe_attention_decode``).

``run`` computes a case either through the package (``own``) or in its plain form: elementary torch operations in 32 bits, the
positions' angles in 64, one rounding at the end.  ``exact`` is the definition in 64 bits.

Head counts and head dimensions are those of layers of the repository's workloads (d_model 1024 as 16 heads of 64, 768 as 12
of 64, 2048 as 16 of 128, 4096 as 32 of 128 with 8 key-value heads) and generic ones.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
ES = {"bf16": 2, "f32": 4}


# ---- cases ------------------------------------------------------------------------------------------

def _attend(name, **kw):
    c = dict(op="attend", B=1, hq=16, hkv=16, D=64, page=16, layout="token", dtype="bf16", lo=1, hi=128, empty=False, spare=0,
             cap=0.0, window=0, slopes=False, lse=False)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def _append(name, **kw):
    c = dict(op="append", T=1, seqs=1, start=0, hq=16, hkv=16, D=64, R=64, axes=1, inter=False, page=16, layout="token", dtype="bf16")
    c.update(kw)
    if name:
        c["name"] = name
    return c


def _rotary(name, **kw):
    c = dict(op="rotary", T=1, H=16, D=64, R=64, axes=1, inter=False, inverse=False, fused=False, start=0, dtype="bf16")
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one request, a short prompt, a layer of the GPT-style model: the smallest call, launches and latency
        _attend("attend_one", hi=173, lo=173),
        # one request with a very long context, grouped heads, head-major pages: only the length can fill the machine
        _attend("attend_long", hq=32, hkv=8, D=128, page=64, layout="head", lo=131071, hi=131071, lse=True),
        # a serving batch in the midst of its conversations: ragged lengths, small pages
        _attend("attend_batch", B=64, hq=32, hkv=8, D=128, lo=100, hi=8192),
        # a layer that attends to a window only, capped scores, wide heads; some places of the batch are empty
        _attend("attend_window", B=96, hq=16, hkv=2, D=256, page=32, layout="head", lo=1, hi=16384, empty=True, cap=50.0, window=1025),
        # float32 run of a model with distance biases (reference outputs, a probe model), pages that fit no tile
        _attend("attend_f32", B=13, hq=12, hkv=12, D=64, page=20, lo=7, hi=2000, dtype="f32", slopes=True, lse=True),
        # the largest step: a full server, eight queries per key head
        _attend("attend_full", B=256, hq=64, hkv=8, D=128, page=64, lo=2048, hi=14336),
        # one request's new token
        _append("append_one", start=172),
        # a serving batch's new tokens, each into its own sequence
        _append("append_batch", T=256, seqs=256, start=4097, hq=32, hkv=8, D=128, R=128),
        # prompts of five requests at once, an image among them: three axes
        _append("append_prompt", T=16389, seqs=5, start=0, hq=32, hkv=8, D=128, R=128, axes=3, page=64, layout="head"),
        # float32 queries of a small model, interleaved pairs
        _rotary("rotary_f32", T=1000, H=12, inter=True, dtype="f32"),
        # queries of images and video in training: three axes, read out of the fused projection's output
        _rotary("rotary_video", T=8192, H=16, axes=3, fused=True),
        # gradient of a long context's queries, only half of each head rotated
        _rotary("rotary_back", T=32768, H=32, D=128, R=64, inverse=True, start=100000),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _heads(rng):
    D = rng.choice([64, 64, 80, 96, 128, 128, 128, 192, 256])
    hkv = rng.choice([1, 2, 4, 5, 8, 12, 16])
    return D, hkv, hkv * rng.choice([1, 1, 2, 3, 4, 6, 8, 16])


def _axes(rng, D):
    R = rng.choice([D, D, D // 2])
    return dict(R=R, axes=rng.choice([1, 1, 3]), inter=rng.random() < 0.3)


def draw(rng):
    op = rng.choice(["attend", "attend", "append", "rotary"])
    D, hkv, hq = _heads(rng)
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    page = rng.choice([1, 16, 16, 20, 32, 64, 100, 128, 256])
    layout = rng.choice(["token", "head"])
    if op == "attend":
        hi = _log(rng, 1, 131072)
        limit = 6.0e9 / (4.0 * hkv * D * ES[dtype] * hi)  # half the largest listed case's keys and values, at most
        B = min(_log(rng, 1, 512), max(1, int(limit)))
        lo = rng.choice([hi, max(1, hi // 2), 1])
        return _attend(None, B=B, hq=hq, hkv=hkv, D=D, page=page, layout=layout, dtype=dtype, lo=lo, hi=hi, empty=B > 1 and rng.random() < 0.3,
                       spare=rng.choice([0, 0, 3, 1000]), cap=rng.choice([0.0, 0.0, 30.0]), slopes=rng.random() < 0.25, lse=rng.random() < 0.4,
                       window=rng.choice([0, 0, 0, 1, 100, 1000, 4096]))
    if op == "append":
        T = _log(rng, 1, min(65536, int(16389 * 48 * 128 * 2 / ((hq + 2 * hkv) * D * ES[dtype]))))
        return _append(None, T=T, seqs=rng.choice([1, T, min(T, 5)]) if T <= 512 else rng.choice([1, 5, 32]), start=rng.choice([0, 77, _log(rng, 1, 8000)]),
                       hq=hq, hkv=hkv, D=D, page=page, layout=layout, dtype=dtype, **_axes(rng, D))
    T = _log(rng, 1, min(65536, int(32768 * 32 * 128 * 2 / (hq * D * ES[dtype]))))
    return _rotary(None, T=T, H=hq, D=D, inverse=rng.random() < 0.4, fused=rng.random() < 0.5, start=rng.choice([0, 0, 1000000]), dtype=dtype, **_axes(rng, D))


# ---- inputs -----------------------------------------------------------------------------------------

def _lens(c):
    """Lengths of the batch's sequences: the first has the longest, the others are spread over lo..hi."""
    r = random.Random(c["B"] * 1000003 + c["hi"] * 17 + c["lo"])
    lens = [c["hi"]] + [r.randint(c["lo"], c["hi"]) for _ in range(c["B"] - 1)]
    if c["empty"]:
        for b in range(1, c["B"], 7):
            lens[b] = 0
    return lens


def _counts(c):
    """New tokens of each sequence of an append: a token each, or prompts of uneven lengths."""
    T, S = c["T"], c["seqs"]
    if T == S:
        return [1] * S
    w = [1 + (i * 7919) % 13 for i in range(S)]
    n = [T * x // sum(w) for x in w]
    n[0] += T - sum(n)
    return n


def _gen(seed, salt):
    return torch.Generator(device="cuda").manual_seed(seed * 7 + salt)


def _pages(c, widths, seed):
    """Page table [sequences, widest] over a pool in random order (entries past a sequence's own are -1) and the pool's size."""
    total, width = sum(widths), max(max(widths), 1) + c.get("spare", 0)
    n_pages = max(total, 1) + 3
    order = torch.randperm(n_pages, device="cuda", generator=_gen(seed, 1)).to(torch.int32)
    first = torch.tensor([0] + widths[:-1]).cumsum(0).cuda()[:, None]
    at = torch.arange(width, device="cuda")[None, :]
    has = at < torch.tensor(widths).cuda()[:, None]
    return torch.where(has, order[(first + at).clamp(max=n_pages - 1)], -1).to(torch.int32).contiguous(), n_pages


def _pool(c, n_pages, seed, salt):
    mid = (c["page"], c["hkv"]) if c["layout"] == "token" else (c["hkv"], c["page"])
    return torch.empty((n_pages,) + mid + (c["D"],), dtype=DT[c["dtype"]], device="cuda").normal_(generator=_gen(seed, salt))


def _freqs(c):
    """Radians per position of every pair: each axis has its own geometric series (base 10000), and how many pairs an axis has."""
    half = c["R"] // 2
    if c["axes"] == 1:
        parts = [half]
    else:
        parts = [half // 4, (half - half // 4) // 2]
        parts.append(half - sum(parts))
    f = [10000.0 ** (-i / n) for n in parts for i in range(n)]
    return torch.tensor(f, dtype=torch.float64, device="cuda"), tuple(parts)


def _positions(c, places):
    """int32 [axes, T]: the places themselves, or (time, height, width) of pictures of 24 x 32 patches."""
    if c["axes"] == 1:
        return places[None].contiguous()
    return torch.stack([places // 768, places // 32 % 24, places % 32]).to(torch.int32).contiguous()


def _inputs(c, seed):
    s = {}
    dt, D = DT[c["dtype"]], c["D"]
    if c["op"] == "attend":
        lens = _lens(c)
        s["table"], n = _pages(c, [-(-x // c["page"]) for x in lens], seed)
        s["k"], s["v"] = _pool(c, n, seed, 2), _pool(c, n, seed, 3)
        s["q"] = (2.0 * torch.randn(c["B"], c["hq"], D, device="cuda", generator=_gen(seed, 4))).to(dt)
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        if c["slopes"]:
            s["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / c["hq"]) for h in range(c["hq"])], dtype=torch.float32, device="cuda")
    elif c["op"] == "append":
        n_new, T = _counts(c), c["T"]
        s["table"], n = _pages(c, [-(-(c["start"] + x) // c["page"]) for x in n_new], seed)
        s["k"], s["v"] = _pool(c, n, seed, 2), _pool(c, n, seed, 3)
        # one projection's output holds the queries, keys and values of a token side by side
        qkv = torch.randn(T, c["hq"] + 2 * c["hkv"], D, device="cuda", generator=_gen(seed, 4)).to(dt)
        s["q"], s["k_new"], s["v_new"] = qkv[:, :c["hq"]], qkv[:, c["hq"]:c["hq"] + c["hkv"]], qkv[:, c["hq"] + c["hkv"]:]
        s["seq"] = torch.repeat_interleave(torch.arange(c["seqs"]), torch.tensor(n_new)).to(torch.int32).cuda()
        s["place"] = torch.cat([torch.arange(c["start"], c["start"] + x) for x in n_new]).to(torch.int32).cuda()
        s["pos"] = _positions(c, s["place"])
    else:
        x = torch.randn(c["T"], c["H"] * (3 if c["fused"] else 1), D, device="cuda", generator=_gen(seed, 4)).to(dt)
        s["x"] = x[:, :c["H"]]
        s["pos"] = _positions(c, c["start"] + torch.arange(c["T"], dtype=torch.int32, device="cuda"))
    if "R" in c:
        s["freqs"], s["parts"] = _freqs(c)
        s["axis"] = torch.tensor([a for a, n in enumerate(s["parts"]) for _ in range(n)], device="cuda")
    return s


def prepare(case, seed):
    c = case
    s = _inputs(c, seed)
    s["case"] = c
    if c["op"] == "attend":
        s["host_lens"] = _lens(c)
        s["out"] = torch.empty_like(s["q"])
        s["out_lse"] = torch.empty(c["B"], c["hq"], dtype=torch.float32, device="cuda") if c["lse"] else None
    elif c["op"] == "append":
        s["q_out"] = torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda")
    else:
        s["out"] = torch.empty(s["x"].shape, dtype=s["x"].dtype, device="cuda")
    if own:
        import paper_2205_10034_amd as M
        if "R" in c:
            s["rotary"] = M.Rotary(c["D"], s["freqs"], axis_pairs=s["parts"], interleaved=c["inter"])
        if c["op"] != "rotary":
            s["cache"] = M.KVCache(s["k"], s["v"], s["table"], layout=c["layout"] + "_major")
        if c["op"] == "attend":
            s["ws"] = torch.empty(M.moe_attention_decode_workspace_bytes(s["cache"], c["hq"]), dtype=torch.uint8, device="cuda")
    return s


# ---- the operators ----------------------------------------------------------------------------------

def run(state):
    c = state["case"]
    if own:
        return _run_own(c, state)
    return {"attend": _plain_attend, "append": _plain_append, "rotary": _plain_rotary}[c["op"]](c, state)


def _run_own(c, s):
    import paper_2205_10034_amd as M
    if c["op"] == "attend":
        M.moe_attention_decode(s["cache"], s["q"], s["lens"], s["out"], s["ws"], softcap=c["cap"], window=c["window"], slopes=s.get("slopes"), lse=s["out_lse"])
        return [s["out"], s["out_lse"]] if c["lse"] else [s["out"]]
    if c["op"] == "append":
        M.moe_kv_append(s["cache"], s["k_new"], s["v_new"], s["place"], token_seq=s["seq"], rotary=s["rotary"], positions=s["pos"], q=s["q"], q_out=s["q_out"])
        return [s["k"], s["v"], s["q_out"]]
    M.moe_rotary(s["rotary"], s["x"], s["pos"], s["out"], inverse=c["inverse"])
    return [s["out"]]


def _turn(x, cos, sin, R, inter):
    """x [T, H, D] in 32 bits, its first R dimensions rotated by the angles of cos, sin [T, 1, R/2]."""
    head, rest = x[..., :R], x[..., R:]
    u, v = (head[..., 0::2], head[..., 1::2]) if inter else (head[..., :R // 2], head[..., R // 2:])
    a, b = u * cos - v * sin, u * sin + v * cos
    return torch.cat([torch.stack([a, b], -1).flatten(-2) if inter else torch.cat([a, b], -1), rest], -1)


def _angles(c, s, inverse=False):
    a = s["pos"][s["axis"]].t().double() * s["freqs"]
    sin = torch.sin(a)
    return torch.cos(a).float()[:, None], (-sin if inverse else sin).float()[:, None]


def _plain_rotary(c, s):
    cos, sin = _angles(c, s, c["inverse"])
    s["out"].copy_(_turn(s["x"].float(), cos, sin, c["R"], c["inter"]))
    return [s["out"]]


def _plain_append(c, s):
    cos, sin = _angles(c, s)
    dt = DT[c["dtype"]]
    place = s["place"].long()
    page = s["table"][s["seq"].long(), place // c["page"]].long()
    row = place % c["page"]
    k, v = _turn(s["k_new"].float(), cos, sin, c["R"], c["inter"]).to(dt), s["v_new"]
    if c["layout"] == "token":
        s["k"][page, row], s["v"][page, row] = k, v
    else:
        s["k"][page, :, row], s["v"][page, :, row] = k, v
    s["q_out"].copy_(_turn(s["q"].float(), cos, sin, c["R"], c["inter"]))
    return [s["k"], s["v"], s["q_out"]]


def _groups(c, lens, budget):
    """Runs of sequences whose keys, padded to the pages of the longest (a window's: to those it can touch), stay below budget
    elements."""
    P = c["page"]
    most = -(-c["window"] // P) + 1 if c["window"] else 1 << 40
    first = 0
    while first < len(lens):
        n, pages = 0, 1
        while first + n < len(lens):
            more = max(pages, min(most, -(-lens[first + n] // P)))
            if n and (n + 1) * more * P * c["hkv"] * c["D"] > budget:
                break
            n, pages = n + 1, more
        yield first, first + n, pages
        first += n


def _plain_attend(c, s):
    G, D, P = c["hq"] // c["hkv"], c["D"], c["page"]
    for b0, b1, n_pages in _groups(c, s["host_lens"], 1 << 28):
        B = b1 - b0
        n = s["lens"][b0:b1, None]
        first = torch.div((n - c["window"]).clamp(min=0), P, rounding_mode="floor") if c["window"] else torch.zeros_like(n)
        at = first * P + torch.arange(n_pages * P, device="cuda")[None, :]
        keep = at < n
        if c["window"]:
            keep = keep & (n - at <= c["window"])
        column = first + torch.arange(n_pages, device="cuda")[None, :]
        table = torch.gather(s["table"][b0:b1].long(), 1, column.long().clamp(max=s["table"].shape[1] - 1)).clamp(min=0)

        def rows(pool):
            x = pool[table]
            if c["layout"] == "head":
                x = x.transpose(2, 3)
            return x.reshape(B, n_pages * P, c["hkv"], D).float().transpose(1, 2)

        z = torch.matmul(s["q"][b0:b1].float().view(B, c["hkv"], G, D), rows(s["k"]).transpose(2, 3)) * (D ** -0.5)
        if c["cap"]:
            z = torch.tanh(z / c["cap"]) * c["cap"]
        if c["slopes"]:
            z = z - s["slopes"].view(1, c["hkv"], G, 1) * (n - 1 - at)[:, None, None].float()
        z = torch.where(keep[:, None, None], z, float("-inf"))
        top = z.amax(-1, keepdim=True)
        p = torch.exp(z - torch.where(top == float("-inf"), 0.0, top))
        total = p.sum(-1, keepdim=True)
        o = torch.matmul(p, rows(s["v"])) / torch.where(total > 0, total, 1.0)
        s["out"][b0:b1] = o.reshape(B, c["hq"], D)
        if c["lse"]:
            s["out_lse"][b0:b1] = (torch.log(total) + top).reshape(B, c["hq"])
    return [s["out"], s["out_lse"]] if c["lse"] else [s["out"]]


# ---- what a pass cannot do without --------------------------------------------------------------------

def work(case):
    c = case
    es = ES[c["dtype"]]
    if c["op"] == "attend":
        keys = sum(min(n, c["window"]) if c["window"] else n for n in _lens(c))
        return {"bytes": 2 * keys * c["hkv"] * c["D"] * es + 2 * c["B"] * c["hq"] * c["D"] * es + (4 * c["B"] * c["hq"] if c["lse"] else 0),
                "flops": 4 * keys * c["hq"] * c["D"]}
    if c["op"] == "append":
        return {"bytes": 2 * c["T"] * (c["hq"] + 2 * c["hkv"]) * c["D"] * es + 4 * c["T"] * (2 + c["axes"]),
                "flops": 3 * c["T"] * (c["hq"] + c["hkv"]) * c["R"]}
    return {"bytes": 2 * c["T"] * c["H"] * c["D"] * es + 4 * c["T"] * c["axes"], "flops": 3 * c["T"] * c["H"] * c["R"]}


# ---- the definition in 64 bits ------------------------------------------------------------------------

def _exact_rotated(c, s, x, sign):
    """Each pair as a complex number times exp(i angle)."""
    half = c["R"] // 2
    axis = [a for a, n in enumerate(s["parts"]) for _ in range(n)]
    angle = torch.stack([s["pos"][a].double() * f for a, f in zip(axis, s["freqs"].tolist())], -1)
    spin = torch.polar(torch.ones_like(angle), sign * angle)[:, None, :]
    y = x.double()
    i = torch.arange(half, device="cuda")
    lo, hi = (2 * i, 2 * i + 1) if c["inter"] else (i, i + half)
    z = torch.complex(y[:, :, lo], y[:, :, hi]) * spin
    y[:, :, lo], y[:, :, hi] = z.real, z.imag
    return y


def exact(case, seed):
    c = case
    s = _inputs(c, seed)
    if c["op"] == "rotary":
        return [_exact_rotated(c, s, s["x"].float(), -1.0 if c["inverse"] else 1.0)]
    if c["op"] == "append":
        k, v = s["k"].double(), s["v"].double()
        rows_k = _exact_rotated(c, s, s["k_new"].float(), 1.0)
        # the pool seen as [page, place, head, dim] whatever its layout
        kk, vv = (k, v) if c["layout"] == "token" else (k.permute(0, 2, 1, 3), v.permute(0, 2, 1, 3))
        flat = s["table"].flatten()[s["seq"].long() * s["table"].shape[1] + torch.div(s["place"], c["page"], rounding_mode="floor").long()].long()
        kk[flat, (s["place"] % c["page"]).long()] = rows_k
        vv[flat, (s["place"] % c["page"]).long()] = s["v_new"].double()
        return [k, v, _exact_rotated(c, s, s["q"].float(), 1.0)]
    G, D, lens = c["hq"] // c["hkv"], c["D"], _lens(c)
    out = torch.zeros(c["B"], c["hq"], D, dtype=torch.float64, device="cuda")
    lse = torch.full((c["B"], c["hq"]), float("-inf"), dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        if n == 0:
            continue
        first = max(0, n - c["window"]) if c["window"] else 0
        j = torch.arange(first, n, device="cuda")
        page, row = s["table"][b][j // c["page"]].long(), j % c["page"]
        for h in range(c["hkv"]):
            k, v = (s["k"][page, row, h], s["v"][page, row, h]) if c["layout"] == "token" else (s["k"][page, h, row], s["v"][page, h, row])
            z = (k.double() @ s["q"][b, h * G:(h + 1) * G].double().t()) / math.sqrt(D)
            if c["cap"]:
                z = c["cap"] * torch.tanh(z / c["cap"])
            if c["slopes"]:
                z = z - (n - 1 - j)[:, None].double() * s["slopes"][h * G:(h + 1) * G].double()[None]
            lse[b, h * G:(h + 1) * G] = torch.logsumexp(z, 0)
            out[b, h * G:(h + 1) * G] = torch.softmax(z, 0).t() @ v.double()
    return [out, lse] if c["lse"] else [out]
