"""Plain 64-bit forms of the 8-bit cache, and batches whose requests share prefixes."""
import numpy as np
import torch

from paged_ref import DT, ints

# every e4m3 number from 0 to 448, by its code
GRID = np.array([(1 + f / 8) * 2.0 ** (e - 7) if e else f / 8 * 2.0 ** -6 for e in range(16) for f in range(8)][:127])


def values(codes, exponents, which, page_ids=None):
    """What an 8-bit cache [n_pages, page, Hkv, d] holds, in 64 bits (numpy); NaN codes NaN."""
    bits = codes.view(torch.uint8).cpu().numpy()
    x = np.append(GRID, np.nan)[bits & 127] * np.where(bits & 128, -1.0, 1.0)
    power = np.exp2(np.clip(exponents.cpu().numpy()[..., which].astype(np.float64), 1, 254) - 127)
    return x * power.transpose(0, 2, 1)[..., None]


def quantise(x):
    """x [..., d] in 64 bits, numpy: (the nearest e4m3 multiples of the rows' powers of two, the powers' bytes); no number at all: NaN."""
    fine = np.isfinite(x)
    size = np.where(fine, np.abs(x), 0.0)
    top = size.max(-1, keepdims=True)
    power = np.full_like(top, 2.0 ** -100)
    for e in range(-99, 121):                                # the smallest power of two that holds the row
        power = np.where(top > 448 * power, 2.0 ** e, power)
    y = size / power
    hi = np.clip(np.searchsorted(GRID, y), 1, 126)
    lo = hi - 1
    below, above = y - GRID[lo], GRID[hi] - y
    pick = np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    out = np.copysign(GRID[pick] * power, x)
    return np.where(fine, out, np.nan), (np.log2(power)[..., 0] + 127).astype(np.uint8)


def wide_table(B, Hkv, d, page):
    """Entries per request for which prefixes are read once, whatever the types: 200 MiB of one byte per element."""
    return (200 << 20) // (B * page * 2 * Hkv * d) + 1


class Shared:
    """Requests whose tokens are kv, the last `new` of them new, on pages: groups = [(first request, end, shared tokens)].  cache: "e4m3" or
    "own" (of dtype).  What no row may see is NaN, its powers any bytes; table entries behind a request's pages are no pages at all; wide: with groups, tables
    so wide that prefixes are read once for them."""

    def __init__(self, kv, new, groups=(), dtype="bf16", cache="own", Hq=4, Hkv=2, d=64, page=16, layout="token", seed=0, extra_rows=0, width=None,
                 q_gain=1.0, row_gap=0, device="cuda", wide=True):
        g = torch.Generator(device=device).manual_seed(seed)
        rnd = lambda *s: torch.randn(s, generator=g, device=device)       # noqa: E731
        self.kv, self.new, self.groups = list(kv), list(new), list(groups)
        self.dtype, self.cache, self.Hq, self.Hkv, self.d, self.page = dtype, cache, Hq, Hkv, d, page
        B = len(kv)
        shared = [0] * B
        for a, e, p in groups:
            for b in range(a + 1, e):
                shared[b] = min(p, kv[a], kv[b]) // page     # whole pages of the group's first request
        held = [-(-k // page) for k in kv]
        width = width or max(max(held), 1)
        if groups and wide:                  # (where the tables could hold little, nothing is shared)
            width = max(width, wide_table(B, Hkv, d, page))
        n_pages = sum(held) + 2
        kind = torch.float8_e4m3fn if cache == "e4m3" else DT[dtype]
        shape = (n_pages, Hkv, page, d) if layout == "head" else (n_pages, page, Hkv, d)
        if cache == "e4m3":
            caches = [torch.full(shape, 0x7f, dtype=torch.uint8, device=device).view(kind) for _ in range(2)]
            self.exps = torch.randint(0, 256, (n_pages, Hkv, page, 2), generator=g, device=device, dtype=torch.uint8)
        else:
            caches = [torch.full(shape, float("nan"), dtype=kind, device=device) for _ in range(2)]
            self.exps = None
        self.k, self.v = (c.permute(0, 2, 1, 3) if layout == "head" else c for c in caches)
        ids = torch.randperm(n_pages, generator=g, device=device)
        self.table = torch.full((B, width), -1, dtype=torch.int32, device=device)
        self.table[:, ::2] = 1 << 30
        self.K, self.V, at = [], [], 0
        prefix = {a: [rnd(p, Hkv, d), rnd(p, Hkv, d), torch.randint(117, 123, (p, Hkv, 2), generator=g, device=device, dtype=torch.uint8)]
                  for a, e, p in groups}
        for b in range(B):
            own = ids[at:at + held[b]].clone()
            at += held[b]
            a = next((a for a, e, p in groups if a <= b < e), b)
            if shared[b]:
                own[:shared[b]] = self.table[a, :shared[b]].long()
            self.table[b, :held[b]] = own.to(torch.int32)
            t = torch.arange(kv[b], device=device)
            power = torch.randint(117, 123, (kv[b], Hkv, 2), generator=g, device=device, dtype=torch.uint8)
            rows = [rnd(kv[b], Hkv, d), rnd(kv[b], Hkv, d)]
            if a in prefix:
                n = min(len(prefix[a][0]), kv[b])
                for w in range(2):
                    rows[w][:n] = prefix[a][w][:n]
                power[:n] = prefix[a][2][:n]
            for w, (cache_, mine) in enumerate(((self.k, self.K), (self.v, self.V))):
                if cache == "e4m3":
                    codes = (rows[w] * 110).clamp(-448, 448).to(kind)
                    cache_.view(torch.uint8)[own[t // page], t % page] = codes.view(torch.uint8)
                    self.exps[own[t // page], :, t % page, w] = power[..., w]
                    mine.append((codes.float() * torch.exp2(power[..., w].float() - 127)[..., None]).to(DT[dtype]))
                else:
                    cache_[own[t // page], t % page] = rows[w].to(kind)
                    mine.append(rows[w].to(kind))
        self.kv_len = ints(kv, device)
        self.cu_host = [0] + np.cumsum(new).tolist()
        self.cu = ints(self.cu_host, device)
        rows = sum(new) + extra_rows
        self.q = (rnd(rows, Hq + row_gap, d) * q_gain).to(DT[dtype])[:, :Hq]
        self.max_new = max(max(new), 1)
        # groups lie side by side: requests between them share nothing
        edges = sorted({0, B} | {a for a, _, _ in groups} | {e for _, e, _ in groups}) if groups else []
        self.start = ints(edges, device) if groups else None
        self.prefix = ints([next((p for a, e, p in groups if (a, e) == (x, y)), 0) for x, y in zip(edges, edges[1:])], device) if groups else None

    def put(self, b, t, K=None, V=None):
        """Other contents of token t of request b, an element's for the whole row (8 bits: NaN alone)."""
        page = self.table[b, t // self.page].long()
        for cache, mine, x in ((self.k, self.K, K), (self.v, self.V, V)):
            if x is not None:
                if self.cache == "e4m3":
                    cache.view(torch.uint8)[page, t % self.page] = 0xff
                else:
                    cache[page, t % self.page] = x
                for c in range(len(self.kv)):
                    if t < self.kv[c] and int(self.table[c, t // self.page]) == int(page):
                        mine[c][t] = x

    def attend(self, sp, groups=True, **kw):
        """The attention through the operator that the batch is for."""
        if not groups:
            return sp.chunk_attn8(self.q, self.k, self.v, self.exps, self.table, self.cu, self.kv_len, self.max_new, **kw)
        return sp.prefix_attn(self.q, self.k, self.v, self.table, self.cu, self.kv_len, self.start, self.prefix, self.max_new,
                              exponents=self.exps, **kw)
