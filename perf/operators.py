"""Operators of a target model served over a paged cache, as cases to be measured: block tables and slot
maps (page_update), rotary positions with several axes (mrope_table, mrope_append) and the attention of new
tokens over the paged cache (chunk_attn).

A case is a dict of plain values.  "op" names the operator; lengths that differ between the requests of a
batch are drawn from "shape", so that work() knows them without a GPU.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ESIZE = {"f32": 4, "bf16": 2}

# heads and head size of the benchmark's model
BASE = {"dtype": "bf16", "Hq": 28, "Hkv": 4, "d": 128}


def listed():
    return [
        # a decoding batch: one new token per request, contexts from short chats to a short video
        {"name": "attn_decode_batch48", "op": "attn", **BASE, "B": 48, "page": 16, "ctx": 8192, "ragged": 1, "new": 1, "mixed": 0,
         "layout": "token", "shape": 1},
        # one request answering about a long video, one token: latency
        {"name": "attn_one_token_26k", "op": "attn", **BASE, "B": 1, "page": 64, "ctx": 26112, "ragged": 0, "new": 1, "mixed": 0,
         "layout": "head", "shape": 2},
        # the last chunk of a long video's prompt, prefilled 2,048 tokens at a time
        {"name": "attn_chunk2048_26k", "op": "attn", **BASE, "B": 1, "page": 64, "ctx": 26112, "ragged": 0, "new": 2048, "mixed": 0,
         "layout": "head", "shape": 3},
        # a whole prompt of odd length at once
        {"name": "attn_prompt_7001", "op": "attn", **BASE, "B": 1, "page": 16, "ctx": 7001, "ragged": 0, "new": 7001, "mixed": 0,
         "layout": "token", "shape": 4},
        # one prompt's chunk rides along with a decoding batch; another head grouping and head size
        {"name": "attn_mixed9_heads64", "op": "attn", "dtype": "bf16", "Hq": 32, "Hkv": 8, "d": 64, "B": 9, "page": 32, "ctx": 5000,
         "ragged": 1, "new": 777, "mixed": 1, "layout": "token", "shape": 5},
        # the tiny fp32 configuration: three requests, five new tokens each
        {"name": "attn_tiny_f32", "op": "attn", "dtype": "f32", "Hq": 4, "Hkv": 1, "d": 64, "B": 3, "page": 16, "ctx": 515, "ragged": 1,
         "new": 5, "mixed": 0, "layout": "token", "shape": 6},
        # a prefill chunk's rows, slices of one fused QKV product, into the cache
        {"name": "append_chunk_8192", "op": "append", **BASE, "rows": 8192, "page": 16, "far": 0, "fused": 1, "layout": "head",
         "shape": 7},
        # a small decoding batch in fp32, far into long contexts
        {"name": "append_step13_f32", "op": "append", "dtype": "f32", "Hq": 16, "Hkv": 4, "d": 64, "rows": 13, "page": 64, "far": 1,
         "fused": 0, "layout": "token", "shape": 8},
        # the table rows of one drafting step
        {"name": "table_step_6", "op": "table", "d": 64, "rows": 6, "far": 1, "shape": 9},
        # the table of a whole long video
        {"name": "table_video_26112", "op": "table", "d": 128, "rows": 26112, "far": 0, "shape": 10},
        # a speculative step of a batch: room for 8 draft rows per request, all rolled back
        {"name": "pages_step_48x8", "op": "pages", "B": 48, "page": 16, "ctx": 8192, "new": 8, "shape": 11},
        # prompts admitted and, at the end, given back
        {"name": "pages_admit_31_prompts", "op": "pages", "B": 31, "page": 16, "ctx": 0, "new": 1500, "shape": 12},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "attn", "attn", "append", "table", "pages"])
    shape = rng.randrange(1 << 30)
    if op == "pages":
        return {"op": op, "B": _log(rng, 1, 64), "page": rng.choice([16, 32, 64]), "ctx": rng.choice([0, _log(rng, 1, 8192)]),
                "new": _log(rng, 1, 1000), "shape": shape}
    if op == "table":
        return {"op": op, "d": rng.choice([64, 128]), "rows": _log(rng, 1, 26112), "far": rng.randrange(2), "shape": shape}
    hq, hkv = rng.choice([(28, 4), (16, 4), (32, 8), (8, 8), (4, 1), (14, 2)])
    case = {"op": op, "dtype": rng.choice(["bf16", "bf16", "f32"]), "Hq": hq, "Hkv": hkv, "d": rng.choice([64, 128]),
            "page": rng.choice([16, 32, 64, 128]), "layout": rng.choice(["token", "head"]), "shape": shape}
    if op == "append":
        return {**case, "rows": _log(rng, 1, 8192), "far": rng.randrange(2), "fused": rng.randrange(2)}
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


def _old_new(case):
    """Lengths of the requests before and after a page_update that grows them."""
    rng = random.Random(case["shape"])
    old = [round(case["ctx"] * rng.uniform(0.05, 1.0)) for _ in range(case["B"])]
    grow = [case["new"] if case["new"] <= 16 else max(1, round(case["new"] * rng.uniform(0.2, 1.0))) for _ in range(case["B"])]
    return old, [o + g for o, g in zip(old, grow)]


def work(case):
    op = case["op"]
    if op == "attn":
        kv, n = _lengths(case)
        e, Hq, Hkv, d = ESIZE[case["dtype"]], case["Hq"], case["Hkv"], case["d"]
        pairs = sum(m * k - m * (m - 1) // 2 for k, m in zip(kv, n))       # row i of m sees k - m + 1 + i keys
        return {"bytes": 2 * sum(n) * Hq * d * e + 4 * sum(n) * Hq + 2 * sum(kv) * Hkv * d * e, "flops": 4 * Hq * d * pairs}
    if op == "append":
        one = (case["Hq"] + 2 * case["Hkv"]) * case["d"] * ESIZE[case["dtype"]]
        return {"bytes": case["rows"] * (2 * one + 16), "flops": case["rows"] * (case["Hq"] + case["Hkv"]) * case["d"] * 3}
    if op == "table":
        return {"bytes": case["rows"] * (12 + 4 * case["d"]), "flops": case["rows"] * case["d"] * 10}
    old, new = _old_new(case)
    pages = sum(-(-n // case["page"]) - -(-o // case["page"]) for o, n in zip(old, new))
    rows = sum(new) - sum(old)
    return {"bytes": 16 * case["B"] + 4 * case["B"] + 16 * pages + 8 * rows, "flops": 0}


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(g, shape, dtype):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _cache(g, case, n_pages):
    """K and V pages as views [n_pages, page, Hkv, d]: a page's tokens side by side, or a head's."""
    Hkv, d, ps, dt = case["Hkv"], case["d"], case["page"], DTYPES[case["dtype"]]
    if case["layout"] == "head":
        t = _normal(g, (2, n_pages, Hkv, ps, d), dt)
        return t[0].permute(0, 2, 1, 3), t[1].permute(0, 2, 1, 3)
    t = _normal(g, (2, n_pages, ps, Hkv, d), dt)
    return t[0], t[1]


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


def prepare(case, seed):
    g = _gen(seed)
    op = case["op"]
    s = {"case": case}
    if op == "attn":
        kv, n = _lengths(case)
        ps, B = case["page"], case["B"]
        held = [-(-k // ps) for k in kv]
        perm = torch.randperm(sum(held) + 3, generator=g, device="cuda").to(torch.int32)
        table = torch.full((B, max(held)), -1, dtype=torch.int32, device="cuda")
        mask = torch.arange(max(held), device="cuda")[None, :] < _ints(held)[:, None]
        table[mask] = perm[:sum(held)]
        s["k"], s["v"] = _cache(g, case, sum(held) + 3)
        s["table"], s["kv_len"] = table, _ints(kv)
        s["cu"] = _ints(np.concatenate([[0], np.cumsum(n)]).tolist())
        s["max_new"] = max(n)
        s["q"] = _normal(g, (sum(n), case["Hq"], case["d"]), DTYPES[case["dtype"]])
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(s["q"].shape[:2], dtype=torch.float32, device="cuda")
    elif op == "append":
        N, Hq, Hkv, d, ps, dt = case["rows"], case["Hq"], case["Hkv"], case["d"], case["page"], DTYPES[case["dtype"]]
        if case["fused"]:                   # q, k, v are slices of the projection's output
            x = _normal(g, (N, Hq + 2 * Hkv, d), dt)
            s["q"], s["k"], s["v"] = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
        else:
            s["q"], s["k"], s["v"] = (_normal(g, (N, h, d), dt) for h in (Hq, Hkv, Hkv))
        n_pages = -(-N // ps) + 2
        s["kc"], s["vc"] = _cache(g, case, n_pages)
        first = random.Random(seed).randrange(ps)
        at = torch.arange(N, device="cuda") + first          # a sequence's next tokens, on pages in no order
        perm = torch.randperm(n_pages, generator=g, device="cuda")
        s["slots"] = (perm[at // ps] * ps + at % ps).to(torch.int32)
        s["pos"] = _positions(case, seed)
        s["inv"], s["axis"] = _rotary(case)
        s["q_out"] = torch.empty((N, Hq, d), dtype=dt, device="cuda")
    elif op == "table":
        s["pos"] = _positions(case, seed)
        s["inv"], s["axis"] = _rotary(case)
        s["cos"] = torch.empty((case["rows"], case["d"] // 2), dtype=torch.float32, device="cuda")
        s["sin"] = torch.empty_like(s["cos"])
    else:
        old, new = _old_new(case)
        ps = case["page"]
        held = [-(-o // ps) for o in old]
        need = [-(-x // ps) for x in new]
        total = sum(need) + 5
        ids = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
        width = max(need) + 1
        s["table"] = torch.full((len(old), width), -1, dtype=torch.int32, device="cuda")
        s["table"][torch.arange(width, device="cuda")[None, :] < _ints(held)[:, None]] = ids[:sum(held)]
        s["free"] = torch.cat([ids[sum(held):], torch.full((sum(held),), -1, dtype=torch.int32, device="cuda")])
        s["n_free"] = _ints([total - sum(held)])
        s["old"], s["new"], s["rows"] = _ints(old), _ints(new), sum(new) - sum(old)
        s["offset"] = _ints([random.Random(seed + b).randrange(-50, 3) for b in range(len(old))])
    return s


# ------------------------------------------------------------------ plain forms
def _attn(s):
    c = s["case"]
    Hq, Hkv, d = c["Hq"], c["Hkv"], c["d"]
    G, N = Hq // Hkv, s["max_new"]
    table, cu, kv_len = s["table"].long().clamp(min=0), s["cu"].long(), s["kv_len"].long()
    B, W = table.shape
    L = W * c["page"]
    n_new = cu[1:] - cu[:-1]
    i = torch.arange(N, device="cuda")
    rows = (cu[:-1, None] + i).clamp(max=s["q"].shape[0] - 1)                          # [B, N]
    q = s["q"].float()[rows] * (1.0 / math.sqrt(d))
    q = q.view(B, N, Hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, Hkv, N * G, d)
    k = s["k"][table].float().reshape(B, L, Hkv, d).permute(0, 2, 3, 1).contiguous()
    sc = torch.matmul(q, k).view(B, Hkv, N, G, L)
    del k
    pos = (kv_len - n_new)[:, None] + i                                                # [B, N]
    hidden = torch.arange(L, device="cuda") > pos[:, :, None]
    sc.masked_fill_(hidden[:, None, :, None, :], -math.inf)
    m = sc.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = sc.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    v = s["v"][table].float().reshape(B, L, Hkv, d).permute(0, 2, 1, 3).contiguous()
    o = torch.matmul(p.view(B, Hkv, N * G, L), v).view(B, Hkv, N, G, d) / l
    lse = (m + torch.log(l))[..., 0]
    r = torch.arange(s["q"].shape[0], device="cuda")
    b = torch.searchsorted(cu[1:], r, right=True)
    n = r - cu[b]
    out = o.permute(0, 2, 1, 3, 4)[b, n].reshape(-1, Hq, d).to(s["q"].dtype)
    return out, lse.permute(0, 2, 1, 3)[b, n].reshape(-1, Hq)


def _cos_sin(s):
    axis = torch.from_numpy(s["axis"]).long().cuda()
    angle = s["pos"].t().double()[:, axis] * torch.from_numpy(s["inv"]).cuda()         # [N, d/2], 64 bits
    return torch.cos(angle).float(), torch.sin(angle).float()


def _append(s):
    c, s_ = _cos_sin(s)
    c, s_ = c[:, None, :], s_[:, None, :]

    def turn(x):
        a, b = x.float().chunk(2, dim=-1)
        return torch.cat([a * c - b * s_, b * c + a * s_], dim=-1).to(x.dtype)

    page, at = s["slots"].long() // s["case"]["page"], s["slots"].long() % s["case"]["page"]
    s["kc"][page, at] = turn(s["k"])
    s["vc"][page, at] = s["v"]
    return turn(s["q"]), s["kc"], s["vc"]


def _grow(s, old, new, table, free, n_free, rows):
    """The update of block tables, as tensor operations: (slots, cu, positions, table, free, n_free)."""
    ps = s["case"]["page"]
    old, new = old.long(), new.long()
    held, need = (old + ps - 1) // ps, (new + ps - 1) // ps
    j = torch.arange(table.shape[1], device="cuda")[None, :]
    give, take = (held - need).clamp(min=0), (need - held).clamp(min=0)
    top = n_free.long() + give.sum() - 1
    back = (torch.cumsum(give, 0) - give)[:, None] + j - need[:, None]
    gone = (j >= need[:, None]) & (j < held[:, None])
    k = torch.arange(free.shape[0], device="cuda")
    # the k-th page given back lands on stack[top - k]: a scatter through an extra last element
    free = torch.cat([free, free[:1]])
    free[torch.where(gone, top - back, free.shape[0] - 1)] = table
    free = free[:-1]
    got = (torch.cumsum(take, 0) - take)[:, None] + j - held[:, None]
    come = (j >= held[:, None]) & (j < need[:, None])
    table = torch.where(come, free[(top - got).clamp(0, len(k) - 1)], table)
    n_free = (top + 1 - take.sum()).to(torch.int32).view(1)
    n = (new - old).clamp(min=0)
    cu = torch.cat([n.new_zeros(1), torch.cumsum(n, 0)])
    r = torch.arange(rows, device="cuda")
    b = torch.searchsorted(cu[1:], r, right=True)
    at = old[b] + r - cu[b]
    slots = table[b, at // ps].long() * ps + at % ps
    return slots.to(torch.int32), cu.to(torch.int32), (at + s["offset"][b]).to(torch.int32), table, free, n_free


def _pages(s):
    slots, cu, pos, table, free, n_free = _grow(s, s["old"], s["new"], s["table"], s["free"], s["n_free"], s["rows"])
    taken = n_free
    _, _, _, table, free, n_free = _grow(s, s["new"], s["old"], table, free, n_free, 0)
    return slots, cu, pos, taken, table, free, n_free


def run(s):
    op = s["case"]["op"]
    if not own:
        return {"attn": _attn, "append": _append, "table": _cos_sin, "pages": _pages}[op](s)
    import paper_2602_15318_amd as sp
    if op == "attn":
        return sp.chunk_attn(s["q"], s["k"], s["v"], s["table"], s["cu"], s["kv_len"], s["max_new"], out=s["out"], lse=s["lse"])
    if op == "append":
        q = sp.mrope_append(s["q"], s["k"], s["v"], s["pos"], s["inv"], s["axis"], s["slots"], s["kc"], s["vc"], q_out=s["q_out"])
        return q, s["kc"], s["vc"]
    if op == "table":
        return sp.mrope_table(s["pos"], s["inv"], s["axis"], cos=s["cos"], sin=s["sin"])
    ps = s["case"]["page"]
    slots, cu, pos, _ = sp.page_update(s["old"], s["new"], s["table"], s["free"], s["n_free"], ps, s["rows"], pos_offset=s["offset"])
    taken = s["n_free"].clone()
    sp.page_update(s["new"], s["old"], s["table"], s["free"], s["n_free"], ps, 0)
    return slots, cu, pos, taken, s["table"], s["free"], s["n_free"]


# ------------------------------------------------------------------ the definition in 64 bits, row by row
def _exact_attn(case, s):
    kv, n = _lengths(case)
    Hq, Hkv, d, ps = case["Hq"], case["Hkv"], case["d"], case["page"]
    G = Hq // Hkv
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    r0 = 0
    for b in range(case["B"]):
        pages = s["table"][b, :-(-kv[b] // ps)].long()
        k = s["k"][pages].reshape(-1, Hkv, d)[:kv[b]]
        v = s["v"][pages].reshape(-1, Hkv, d)[:kv[b]]
        for i0 in range(0, n[b], 512):
            i1 = min(n[b], i0 + 512)
            seen = kv[b] - n[b] + torch.arange(i0, i1, device="cuda")
            future = torch.arange(kv[b], device="cuda")[None, :] > seen[:, None]
            for h in range(Hq):
                sc = s["q"][r0 + i0:r0 + i1, h].double() @ k[:, h // G].double().t() / math.sqrt(d)
                sc = torch.where(future, -math.inf, sc)
                z = torch.logsumexp(sc, 1)
                lse[r0 + i0:r0 + i1, h] = z
                out[r0 + i0:r0 + i1, h] = torch.exp(sc - z[:, None]) @ v[:, h // G].double()
        r0 += n[b]
    return out, lse


def exact(case, seed):
    op = case["op"]
    if op == "pages":                       # whole numbers only
        return None
    s = prepare(case, seed)
    if op == "attn":
        return _exact_attn(case, s)
    pos = s["pos"].cpu().numpy().astype(np.float64)
    turn = np.exp(1j * np.stack([pos[a] * f for a, f in zip(s["axis"], s["inv"])], axis=1))
    if op == "table":
        return torch.from_numpy(turn.real.copy()).cuda(), torch.from_numpy(turn.imag.copy()).cuda()
    turn = torch.from_numpy(turn).cuda()[:, None, :]
    half = case["d"] // 2
    caches = [s["kc"].double(), s["vc"].double()]
    done = []
    for x in (s["q"], s["k"]):
        z = torch.complex(x[..., :half].double(), x[..., half:].double()) * turn
        done.append(torch.cat([z.real, z.imag], dim=-1))
    for c, x in zip(caches, (done[1], s["v"].double())):
        c[s["slots"].long() // case["page"], s["slots"].long() % case["page"]] = x
    return done[0], caches[0], caches[1]
