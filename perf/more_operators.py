"""Operators for many questions about one long video, as cases to be measured: a paged cache of 8 bits per element that is quantised as
it is written (mrope_append8) and read back (page_gather), attention of new tokens over it (chunk_attn8), and attention of a batch whose
requests share a long prefix, whose keys and values are read once for all of them (prefix_attn).

The 8-bit cache holds, for each (token, KV head) of K and of V, a row of e4m3 codes and a power of two.  With A the largest size in the row
the power is the smallest 2^x with A <= 448 * 2^x (x at least -100), a code the nearest e4m3 number to value / 2^x, ties to even.

A case is a dict of plain values.  "op" names the operator; lengths that differ between the requests of a batch are drawn from "shape", so
that work() knows them without a GPU.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ESIZE = {"f32": 4, "bf16": 2, "e4m3": 1}

# heads and head size of the benchmark's model
BASE = {"dtype": "bf16", "Hq": 28, "Hkv": 4, "d": 128}


def listed():
    return [
        # a prefill chunk's rows, slices of one fused QKV product, into the 8-bit cache, and its keys and values as the cache holds them
        {"name": "append8_chunk_8192", "op": "append8", **BASE, "rows": 8192, "page": 16, "far": 0, "fused": 1, "layout": "head", "shape": 1},
        # a small decoding batch in fp32, far into long contexts
        {"name": "append8_step13_f32", "op": "append8", "dtype": "f32", "Hq": 16, "Hkv": 4, "d": 64, "rows": 13, "page": 64, "far": 1,
         "fused": 0, "layout": "token", "shape": 2},
        # the 8-bit cache of a long video's request laid out for the verification of draft trees, one head after the other
        {"name": "gather_video_26112", "op": "gather", **BASE, "cache": "e4m3", "B": 1, "ctx": 26112, "page": 64, "layout": "head",
         "to": "head", "shape": 3},
        # the last tokens of a few requests out of a cache of the model's own type
        {"name": "gather_tails_7", "op": "gather", "dtype": "bf16", "Hq": 14, "Hkv": 2, "d": 64, "cache": "bf16", "B": 7, "ctx": 333,
         "page": 16, "layout": "token", "to": "token", "shape": 4},
        # a decoding batch: one new token per request, contexts from short chats to a short video
        {"name": "attn8_decode_batch48", "op": "attn8", **BASE, "B": 48, "page": 16, "ctx": 8192, "ragged": 1, "new": 1, "mixed": 0,
         "layout": "token", "shape": 5},
        # one request answering about a long video, one token: latency
        {"name": "attn8_one_token_26k", "op": "attn8", **BASE, "B": 1, "page": 64, "ctx": 26112, "ragged": 0, "new": 1, "mixed": 0,
         "layout": "head", "shape": 6},
        # the last chunk of a long video's prompt, prefilled 2,048 tokens at a time
        {"name": "attn8_chunk2048_26k", "op": "attn8", **BASE, "B": 1, "page": 64, "ctx": 26112, "ragged": 0, "new": 2048, "mixed": 0,
         "layout": "head", "shape": 7},
        # one prompt's chunk rides along with a decoding batch; another head grouping and head size
        {"name": "attn8_mixed9_heads64", "op": "attn8", "dtype": "bf16", "Hq": 32, "Hkv": 8, "d": 64, "B": 9, "page": 32, "ctx": 5000,
         "ragged": 1, "new": 777, "mixed": 1, "layout": "token", "shape": 8},
        # 32 questions about one long video being answered, one token each
        {"name": "prefix_decode32_26k", "op": "prefix", **BASE, "cache": "bf16", "G": 1, "B": 32, "page": 64, "prefix": 26112, "own": 700,
         "new": 1, "ragged_new": 0, "layout": "head", "shape": 9},
        # chains of 8 draft tokens of 12 such requests verified, 8-bit cache, a prefix that ends inside a page
        {"name": "prefix_chains12_8bit", "op": "prefix", **BASE, "cache": "e4m3", "G": 1, "B": 12, "page": 16, "prefix": 17003, "own": 300,
         "new": 8, "ragged_new": 0, "layout": "token", "shape": 10},
        # six questions of up to 200 tokens about a video that has been prefilled, all at once
        {"name": "prefix_questions6_26k", "op": "prefix", **BASE, "cache": "bf16", "G": 1, "B": 6, "page": 64, "prefix": 25600, "own": 200,
         "new": 200, "ragged_new": 1, "layout": "head", "shape": 11},
        # the tiny fp32 configuration: five requests about two images
        {"name": "prefix_two_groups_f32", "op": "prefix", "dtype": "f32", "Hq": 4, "Hkv": 1, "d": 64, "cache": "f32", "G": 2, "B": 5,
         "page": 16, "prefix": 448, "own": 64, "new": 1, "ragged_new": 0, "layout": "token", "shape": 12},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn8", "attn8", "prefix", "prefix", "append8", "gather"])
    hq, hkv = rng.choice([(28, 4), (16, 4), (32, 8), (8, 8), (4, 1), (14, 2)])
    case = {"op": op, "dtype": rng.choice(["bf16", "bf16", "bf16", "f32"]), "Hq": hq, "Hkv": hkv, "d": rng.choice([64, 128]),
            "page": rng.choice([16, 32, 64, 128]), "layout": rng.choice(["token", "head"]), "shape": rng.randrange(1 << 30)}
    if op == "append8":
        return {**case, "rows": _log(rng, 1, 8192), "far": rng.randrange(2), "fused": rng.randrange(2)}
    cache = rng.choice(["e4m3", case["dtype"]])
    if op == "gather":
        return {**case, "cache": cache, "B": _log(rng, 1, 64), "ctx": _log(rng, 1, 8192), "to": rng.choice(["token", "head"])}
    if op == "prefix":
        B, new = rng.choice([(_log(rng, 2, 48), 1), (_log(rng, 2, 12), rng.randint(2, 17)), (rng.randint(2, 6), _log(rng, 18, 200))])
        return {**case, "cache": cache, "G": rng.randint(1, min(3, B)), "B": B, "prefix": _log(rng, 100, 8192), "own": new + _log(rng, 1, 700),
                "new": new, "ragged_new": int(new > 17)}
    kind = rng.choice(["decode", "chain", "chunk", "mixed"])
    if kind == "decode":
        return {**case, "B": _log(rng, 1, 48), "ctx": _log(rng, 1, 8192), "ragged": 1, "new": 1, "mixed": 0}
    if kind == "chain":
        return {**case, "B": _log(rng, 1, 12), "ctx": _log(rng, 20, 8192), "ragged": 1, "new": rng.randint(2, 17), "mixed": 0}
    if kind == "chunk":
        new = _log(rng, 20, 1500)
        return {**case, "B": rng.randint(1, 3), "ctx": new + _log(rng, 1, 6000), "ragged": rng.randrange(2), "new": new, "mixed": 0}
    return {**case, "B": rng.randint(2, 12), "ctx": _log(rng, 500, 5000), "ragged": 1, "new": _log(rng, 20, 500), "mixed": 1}


# ------------------------------------------------------------------ lengths, known without a GPU
def _lengths(case):
    """(tokens in the cache, new ones among them) of every request."""
    rng = random.Random(case["shape"])
    B, ctx, new = case["B"], case["ctx"], case["new"]
    kv = [max(1, round(ctx * rng.uniform(0.05, 1.0))) if case["ragged"] and b else ctx for b in range(B)]
    if case["mixed"]:                       # the first request brings a chunk, the others one token each
        n = [new] + [1] * (B - 1)
    elif case["ragged"] and new > 20:
        n = [new] + [max(1, round(new * rng.uniform(0.3, 1.0))) for _ in range(B - 1)]
    else:
        n = [new] * B
    kv = [max(k, m) for k, m in zip(kv, n)]
    return kv, n


def _shared(case):
    """(first request of every group and the end, prefix of every group, tokens behind the prefix, new ones among them) of a batch in groups."""
    rng = random.Random(case["shape"])
    B, G = case["B"], case["G"]
    start = [0] + sorted(rng.sample(range(1, B), G - 1)) + [B]
    prefix = [case["prefix"]] + [max(1, round(case["prefix"] * rng.uniform(0.3, 1.0))) for _ in range(G - 1)]
    n = [max(1, round(case["new"] * rng.uniform(0.3, 1.0))) if case["ragged_new"] and b else case["new"] for b in range(B)]
    behind = [max(m, round(case["own"] * rng.uniform(0.1, 1.0))) for m in n]
    return start, prefix, behind, n


def _tokens(case):
    """Tokens that a gather reads of every request, and where the first of them is."""
    rng = random.Random(case["shape"])
    first = [rng.randrange(0, 50) if case["B"] > 1 else 0 for _ in range(case["B"])]
    return first, [max(1, round(case["ctx"] * rng.uniform(0.1, 1.0))) if b else case["ctx"] for b in range(case["B"])]


def _pairs(kv, n):
    return sum(m * k - m * (m - 1) // 2 for k, m in zip(kv, n))       # row i of m sees k - m + 1 + i keys


def _row_bytes(case):
    """A token's key or value of one KV head in the cache, its power of two with it."""
    return case["d"] + 1 if case["cache"] == "e4m3" else case["d"] * ESIZE[case["cache"]]


def work(case):
    op, e, Hq, Hkv, d = case["op"], ESIZE[case["dtype"]], case["Hq"], case["Hkv"], case["d"]
    if op == "append8":
        back = 2 * Hkv * d * e
        return {"bytes": case["rows"] * ((2 * Hq + 2 * Hkv) * d * e + 2 * Hkv * (d + 1) + back + 16), "flops": case["rows"] * (Hq + Hkv) * d * 3}
    if op == "gather":
        return {"bytes": sum(_tokens(case)[1]) * 2 * Hkv * (_row_bytes(case) + d * e), "flops": 0}
    if op == "attn8":
        kv, n = _lengths(case)
        return {"bytes": 2 * sum(n) * Hq * d * e + 4 * sum(n) * Hq + 2 * sum(kv) * Hkv * (d + 1), "flops": 4 * Hq * d * _pairs(kv, n)}
    start, prefix, behind, n = _shared(case)
    pairs = _pairs(behind, n) + sum(p * sum(n[a:b]) for p, a, b in zip(prefix, start, start[1:]))
    return {"bytes": 2 * sum(n) * Hq * d * e + 4 * sum(n) * Hq + 2 * (sum(prefix) + sum(behind)) * Hkv * _row_bytes(case), "flops": 4 * Hq * d * pairs}


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(g, shape, dtype):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _cache(g, case, n_pages, kind):
    """K and V pages as views [n_pages, page, Hkv, d]: a page's tokens side by side, or a head's."""
    Hkv, d, ps = case["Hkv"], case["d"], case["page"]
    t = torch.randn((2, n_pages, Hkv, ps, d) if case["layout"] == "head" else (2, n_pages, ps, Hkv, d), generator=g, device="cuda")
    t = t.mul_(110.0).clamp_(-448.0, 448.0).to(torch.float8_e4m3fn) if kind == "e4m3" else t.to(DTYPES[kind])
    if case["layout"] == "head":
        return t[0].permute(0, 2, 1, 3), t[1].permute(0, 2, 1, 3)
    return t[0], t[1]


def _powers(g, case, n_pages):
    """Exponents of the rows' powers of two plus 127, [n_pages, Hkv, page, 2] (K, V): rows of sizes that differ."""
    return torch.randint(118, 122, (n_pages, case["Hkv"], case["page"], 2), generator=g, device="cuda", dtype=torch.uint8)


def _rotary(case):
    """Inverse frequencies (base 1e6) and the axis of each: time, height, width."""
    d = case["d"]
    inv = 1e6 ** (-np.arange(0, d, 2, dtype=np.float64) / d)
    sect = (d // 8, (d // 2 - d // 8) // 2, d // 2 - d // 8 - (d // 2 - d // 8) // 2)
    return inv, np.repeat(np.arange(3, dtype=np.int32), sect)


def _positions(case, seed):
    """[3, N]: a run of text, frames of a grid whose rows and columns count on their own axes, text again."""
    n, rng = case["rows"], random.Random(seed)
    base = rng.randrange(200_000, 1_000_000) if case["far"] else rng.randrange(0, 64)
    text = min(n, 5 + n // 50)
    i = np.arange(n)
    rows, cols = rng.randint(4, 20), rng.randint(4, 24)
    cell = np.maximum(i - text, 0)
    grid = np.stack([cell // (rows * cols), cell // cols % rows, cell % cols]) + text
    p = np.where(i < text, i, grid)
    return torch.from_numpy((p + base).astype(np.int32)).cuda()


def _table(g, held, spare):
    """Block table of requests that hold so many pages each, on pages in no order."""
    perm = torch.randperm(sum(held) + spare, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(held), max(held)), -1, dtype=torch.int32, device="cuda")
    table[torch.arange(max(held), device="cuda")[None, :] < _ints(held)[:, None]] = perm[:sum(held)]
    return table


def prepare(case, seed):
    g = _gen(seed)
    op, ps, Hq, Hkv, d, dt = case["op"], case["page"], case["Hq"], case["Hkv"], case["d"], DTYPES[case["dtype"]]
    s = {"case": case}
    if op == "append8":
        N = case["rows"]
        if case["fused"]:                   # q, k, v are slices of the projection's output
            x = _normal(g, (N, Hq + 2 * Hkv, d), dt)
            s["q"], s["k"], s["v"] = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
        else:
            s["q"], s["k"], s["v"] = (_normal(g, (N, h, d), dt) for h in (Hq, Hkv, Hkv))
        n_pages = -(-N // ps) + 2
        s["kc"], s["vc"] = _cache(g, case, n_pages, "e4m3")
        s["exps"] = _powers(g, case, n_pages)
        first = random.Random(seed).randrange(ps)
        at = torch.arange(N, device="cuda") + first          # a sequence's next tokens, on pages in no order
        perm = torch.randperm(n_pages, generator=g, device="cuda")
        s["slots"] = (perm[at // ps] * ps + at % ps).to(torch.int32)
        s["table"], s["first"], s["cu"] = perm.to(torch.int32).view(1, -1), _ints([first]), _ints([0, N])
        s["pos"] = _positions(case, seed)
        s["inv"], s["axis"] = _rotary(case)
        s["q_out"] = torch.empty((N, Hq, d), dtype=dt, device="cuda")
        s["k_out"], s["v_out"] = (torch.empty((N, Hkv, d), dtype=dt, device="cuda") for _ in range(2))
        return s
    if op == "gather":
        first, n = _tokens(case)
        held = [-(-(f + m) // ps) for f, m in zip(first, n)]
        s["table"], s["first"] = _table(g, held, 2), _ints(first)
        s["cu"], s["rows"] = _ints([0] + np.cumsum(n).tolist()), sum(n)
        n_pages = sum(held) + 2
        shape = (Hkv, sum(n), d) if case["to"] == "head" else (sum(n), Hkv, d)
        s["k_out"], s["v_out"] = (torch.empty(shape, dtype=dt, device="cuda") for _ in range(2))
        if case["to"] == "head":
            s["k_out"], s["v_out"] = s["k_out"].permute(1, 0, 2), s["v_out"].permute(1, 0, 2)
    elif op == "attn8":
        kv, n = _lengths(case)
        held = [-(-k // ps) for k in kv]
        s["table"], n_pages = _table(g, held, 3), sum(held) + 3
    else:
        start, prefix, behind, n = _shared(case)
        of = [max(i for i in range(case["G"]) if start[i] <= b) for b in range(case["B"])]
        kv = [prefix[of[b]] + m for b, m in enumerate(behind)]
        held = [-(-k // ps) for k in kv]
        s["table"], n_pages = _table(g, held, 3), sum(held) + 3
        s["start"], s["prefix"] = _ints(start), _ints(prefix)
    kind = "e4m3" if op == "attn8" else case["cache"]
    s["k"], s["v"] = _cache(g, case, n_pages, kind)
    s["exps"] = _powers(g, case, n_pages) if kind == "e4m3" else None
    if op == "gather":
        return s
    if op == "prefix":                      # whole pages of the prefix are the first request's; the page where it ends is copied
        for i in range(case["G"]):
            a, whole = start[i], prefix[i] // ps
            s["table"][a:start[i + 1], :whole] = s["table"][a, :whole].clone()
            if prefix[i] % ps:
                to, last = s["table"][a:start[i + 1], whole].long(), s["table"][a, whole].long()
                for t in (s["k"], s["v"]):
                    w = t.view(torch.uint8) if kind == "e4m3" else t
                    w[to] = w[last].clone()
                if kind == "e4m3":
                    s["exps"][to] = s["exps"][last].clone()
    s["cu"], s["kv_len"], s["max_new"] = _ints([0] + np.cumsum(n).tolist()), _ints(kv), max(n)
    s["q"] = _normal(g, (sum(n), Hq, d), dt)
    s["out"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty(s["q"].shape[:2], dtype=torch.float32, device="cuda")
    return s


# ------------------------------------------------------------------ plain forms
def _read(s, cache, which, pages):
    """What the cache holds on these pages, [..., page, Hkv, d] in 32 bits."""
    if s["exps"] is None:
        return cache[pages].float()
    codes = cache.view(torch.uint8)[pages].view(torch.float8_e4m3fn).float()
    return codes * torch.exp2(s["exps"][pages][..., which].float() - 127.0).transpose(-1, -2)[..., None]


def _quantise(x):
    """x [..., d] in 64 bits: e4m3 numbers and the exponents of the rows' powers of two."""
    m, e = torch.frexp(x.abs().amax(-1))
    e = torch.where(m > 0.875, e - 8, e - 9).clamp(min=-100)               # 448 is 0.875 * 2^9
    y = torch.ldexp(x, -e[..., None])
    step = torch.exp2((torch.frexp(y)[1] - 1).clamp(min=-6).double() - 3.0)
    return (torch.round(y / step) * step).float(), (e + 127).to(torch.uint8)


def _append(s):
    c = s["case"]
    axis = torch.from_numpy(s["axis"]).long().cuda()
    angle = s["pos"].t().double()[:, axis] * torch.from_numpy(s["inv"]).cuda()         # [N, d/2], 64 bits
    cos, sin = torch.cos(angle)[:, None, :], torch.sin(angle)[:, None, :]

    def turn(x):                            # in 64 bits: a key next to the border of two codes
        a, b = x.double().chunk(2, dim=-1)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)

    page, at = s["slots"].long() // c["page"], s["slots"].long() % c["page"]
    held = []
    for which, (cache, x) in enumerate(((s["kc"], turn(s["k"])), (s["vc"], s["v"].double()))):
        codes, e = _quantise(x)
        cache.view(torch.uint8)[page, at] = codes.to(torch.float8_e4m3fn).view(torch.uint8)
        s["exps"][page, :, at, which] = e
        back = cache.view(torch.uint8)[page, at].view(torch.float8_e4m3fn).float()
        held.append((back * torch.exp2(s["exps"][page, :, at, which].float() - 127.0)[..., None]).to(s["q"].dtype))
    return turn(s["q"]).to(s["q"].dtype), held[0], held[1]


def _gather(s):
    cu, ps = s["cu"].long(), s["case"]["page"]
    r = torch.arange(s["rows"], device="cuda")
    b = torch.searchsorted(cu[1:], r, right=True)
    t = s["first"].long()[b] + r - cu[b]
    page, at = s["table"].long()[b, t // ps], t % ps
    for which, (cache, out) in enumerate(((s["k"], s["k_out"]), (s["v"], s["v_out"]))):
        if s["exps"] is None:
            out.copy_(cache[page, at])
        else:
            codes = cache.view(torch.uint8)[page, at].view(torch.float8_e4m3fn).float()
            out.copy_(codes * torch.exp2(s["exps"][page, :, at, which].float() - 127.0)[..., None])
    return s["k_out"], s["v_out"]


def _attend(q, k, v, hidden):
    """Scaled queries [n, Hkv, rows, g, d] over keys and values [n, L, Hkv, d]; hidden [n, rows, L].  Weighted values, weights' sum, largest score."""
    n, Hkv, rows, g, d = q.shape
    L = k.shape[1]
    sc = torch.matmul(q.reshape(n, Hkv, rows * g, d), k.permute(0, 2, 3, 1).contiguous()).view(n, Hkv, rows, g, L)
    sc.masked_fill_(hidden[:, None, :, None, :], -math.inf)
    m = sc.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = sc.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(n, Hkv, rows * g, L), v.permute(0, 2, 1, 3).contiguous()).view(n, Hkv, rows, g, d)
    return o, l, m


def _queries(s, rows):
    """Scaled queries of rows [n, r] of the batch, [n, Hkv, r, g, d]."""
    c = s["case"]
    q = s["q"].float()[rows.clamp(max=s["q"].shape[0] - 1)] * (1.0 / math.sqrt(c["d"]))
    return q.view(*rows.shape, c["Hkv"], c["Hq"] // c["Hkv"], c["d"]).permute(0, 2, 1, 3, 4)


def _take(x, b, n):
    """Rows n of the requests (or groups) b of [n, Hkv, rows, g, ...] as [rows, Hq, ...]."""
    x = x.permute(0, 2, 1, 3, 4)[b, n]
    return x.reshape(x.shape[0], -1, x.shape[-1])


def _new_rows(s):
    cu = s["cu"].long()
    r = torch.arange(s["q"].shape[0], device="cuda")
    b = torch.searchsorted(cu[1:], r, right=True)
    return cu, r, b


def _attn8(s):
    c = s["case"]
    table, kv_len, N = s["table"].long().clamp(min=0), s["kv_len"].long(), s["max_new"]
    cu, r, b = _new_rows(s)
    i = torch.arange(N, device="cuda")
    L = table.shape[1] * c["page"]
    pos = (kv_len - (cu[1:] - cu[:-1]))[:, None] + i                                   # [B, N]
    k, v = (_read(s, s[x], w, table).reshape(-1, L, c["Hkv"], c["d"]) for w, x in enumerate("kv"))
    o, l, m = _attend(_queries(s, cu[:-1, None] + i), k, v, torch.arange(L, device="cuda") > pos[:, :, None])
    n = r - cu[b]
    return _take(o / l, b, n).to(s["q"].dtype), _take(m + torch.log(l), b, n)[..., 0]


def _prefix(s):
    c = s["case"]
    ps, Hkv, d = c["page"], c["Hkv"], c["d"]
    table, kv_len, N = s["table"].long().clamp(min=0), s["kv_len"].long(), s["max_new"]
    start, prefix = s["start"].long(), s["prefix"].long()
    cu, r, b = _new_rows(s)
    # the prefix, once for all rows of a group
    P = c["prefix"]
    pages = table[start[:-1], :-(-P // ps)]
    k, v = (_read(s, s[x], w, pages).reshape(len(pages), -1, Hkv, d)[:, :P] for w, x in enumerate("kv"))
    row0 = cu[start]
    most = s["q"].shape[0] if c["G"] == 1 else int(s["group_rows"])
    rows = row0[:-1, None] + torch.arange(most, device="cuda")
    hidden = (torch.arange(P, device="cuda") >= prefix[:, None])[:, None, :].expand(-1, most, -1)
    first = _attend(_queries(s, rows), k, v, hidden)
    # what is behind it, request by request
    of = torch.searchsorted(start[1:], torch.arange(c["B"], device="cuda"), right=True)
    own_len = kv_len - prefix[of]
    t = prefix[of][:, None] + torch.arange(s["behind"], device="cuda")
    page = table.gather(1, (t // ps).clamp(max=table.shape[1] - 1))
    k, v = (_at(s, s[x], w, page, t % ps) for w, x in enumerate("kv"))
    i = torch.arange(N, device="cuda")
    pos = (own_len - (cu[1:] - cu[:-1]))[:, None] + i
    then = _attend(_queries(s, cu[:-1, None] + i), k, v, torch.arange(s["behind"], device="cuda") > pos[:, :, None])
    g = torch.searchsorted(row0[1:], r, right=True)
    (o1, l1, m1), (o2, l2, m2) = (_take(x, g, r - row0[g]) for x in first), (_take(x, b, r - cu[b]) for x in then)
    m = torch.maximum(m1, m2)
    f1, f2 = torch.exp(m1 - m), torch.exp(m2 - m)
    l = l1 * f1 + l2 * f2
    return ((o1 * f1 + o2 * f2) / l).to(s["q"].dtype), (m + torch.log(l))[..., 0]


def _at(s, cache, which, page, at):
    """What the cache holds at tokens `at` of pages `page`, [..., Hkv, d] in 32 bits."""
    if s["exps"] is None:
        return cache[page, at].float()
    codes = cache.view(torch.uint8)[page, at].view(torch.float8_e4m3fn).float()
    return codes * torch.exp2(s["exps"][page, :, at, which].float() - 127.0)[..., None]


def run(s):
    op = s["case"]["op"]
    if not own:
        if op == "prefix":                  # sizes of padded arrays, known to a program from its batch
            start, _, behind, n = _shared(s["case"])
            s = {**s, "behind": max(behind), "group_rows": max(sum(n[a:b]) for a, b in zip(start, start[1:]))}
        return {"append8": _append, "gather": _gather, "attn8": _attn8, "prefix": _prefix}[op](s)
    import paper_2602_15318_amd as sp
    if op == "append8":
        q = sp.mrope_append8(s["q"], s["k"], s["v"], s["pos"], s["inv"], s["axis"], s["slots"], s["kc"], s["vc"], s["exps"], q_out=s["q_out"])
        k, v = sp.page_gather(s["kc"], s["vc"], s["table"], s["cu"], s["k_out"], s["v_out"], exponents=s["exps"], first=s["first"])
        return q, k, v
    if op == "gather":
        return sp.page_gather(s["k"], s["v"], s["table"], s["cu"], s["k_out"], s["v_out"], exponents=s["exps"], first=s["first"])
    if op == "attn8":
        return sp.chunk_attn8(s["q"], s["k"], s["v"], s["exps"], s["table"], s["cu"], s["kv_len"], s["max_new"], out=s["out"], lse=s["lse"])
    return sp.prefix_attn(s["q"], s["k"], s["v"], s["table"], s["cu"], s["kv_len"], s["start"], s["prefix"], s["max_new"],
                          exponents=s["exps"], out=s["out"], lse=s["lse"])


# ------------------------------------------------------------------ the definition in 64 bits, row by row
def _value(s, name, which, pages):
    """Keys or values of these pages in 64 bits, [tokens, Hkv, d]."""
    x = s[name]
    if s["exps"] is None:
        return x[pages].double().flatten(0, 1)
    bits = x.view(torch.uint8)[pages].to(torch.int64)
    sign, e, f = bits >> 7, (bits >> 3) & 15, (bits & 7).double()
    size = torch.where(e > 0, torch.ldexp(1.0 + f / 8, e - 7), torch.ldexp(f / 8, torch.full_like(e, -6)))
    power = s["exps"][pages][..., which].to(torch.int64).permute(0, 2, 1)[..., None] - 127
    return torch.ldexp(torch.where(sign == 1, -size, size), power).flatten(0, 1)


def _exact_attn(case, s, kv, n):
    Hq, Hkv, d, ps = case["Hq"], case["Hkv"], case["d"], case["page"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    r0 = 0
    for b in range(case["B"]):
        pages = s["table"][b, :-(-kv[b] // ps)].long()
        k, v = (_value(s, x, w, pages)[:kv[b]] for w, x in enumerate("kv"))
        for i0 in range(0, n[b], 512):
            i1 = min(n[b], i0 + 512)
            seen = kv[b] - n[b] + torch.arange(i0, i1, device="cuda")
            future = torch.arange(kv[b], device="cuda")[None, :] > seen[:, None]
            for h in range(Hq):
                c = h // (Hq // Hkv)
                sc = s["q"][r0 + i0:r0 + i1, h].double() @ k[:, c].t() / math.sqrt(d)
                sc = torch.where(future, -math.inf, sc)
                z = torch.logsumexp(sc, 1)
                lse[r0 + i0:r0 + i1, h] = z
                out[r0 + i0:r0 + i1, h] = torch.exp(sc - z[:, None]) @ v[:, c]
        r0 += n[b]
    return out, lse


def _exact_append(case, s):
    """The rotation as a product of complex numbers, and the nearest of all e4m3 numbers to each element."""
    grid = [(1 + f / 8) * 2.0 ** (e - 7) if e else f / 8 * 2.0 ** -6 for e in range(16) for f in range(8)][:127]
    pos = s["pos"].cpu().numpy().astype(np.float64)
    turn = np.exp(1j * np.stack([pos[a] * f for a, f in zip(s["axis"], s["inv"])], axis=1))[:, None, :]
    half, done = case["d"] // 2, []
    for x, rotated in ((s["q"], True), (s["k"], True), (s["v"], False)):
        x = x.double().cpu().numpy()
        if rotated:
            z = (x[..., :half] + 1j * x[..., half:]) * turn
            x = np.concatenate([z.real, z.imag], axis=-1)
        done.append(x)
    grid = np.array(grid)
    for j in (1, 2):
        x = done[j]
        power = np.exp2(np.maximum(np.ceil(np.log2(np.abs(x).max(-1, keepdims=True) / 448)), -100))
        y = np.abs(x) / power
        hi = np.clip(np.searchsorted(grid, y), 1, 126)
        lo = hi - 1
        below, above = y - grid[lo], grid[hi] - y
        pick = np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
        done[j] = np.copysign(grid[pick] * power, x)
    return tuple(torch.from_numpy(x).cuda() for x in done)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "append8":
        return _exact_append(case, s)
    if op == "gather":
        first, n = _tokens(case)
        held = [[], []]
        for b, (f, m) in enumerate(zip(first, n)):
            pages = s["table"][b, :-(-(f + m) // case["page"])].long()
            for w, x in enumerate("kv"):
                held[w].append(_value(s, x, w, pages)[f:f + m])
        return tuple(torch.cat(x) for x in held)
    if op == "attn8":
        return _exact_attn(case, s, *_lengths(case))
    start, prefix, behind, n = _shared(case)
    return _exact_attn(case, s, s["kv_len"].tolist(), n)
