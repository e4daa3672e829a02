"""Plain 64-bit forms of the paged-cache operators, and inputs for their tests."""
import numpy as np
import torch

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}           # half a step, relative to the value


def ints(x, device="cuda"):
    return torch.tensor(list(x), dtype=torch.int32, device=device)


class Batch:
    """Requests with kv tokens in a paged cache, the last `new` of them new.  Whatever no row may see holds NaN: pages of nobody,
    tails of last pages; entries of the block table behind a request's pages are no pages at all."""

    def __init__(self, kv, new, dtype="bf16", Hq=4, Hkv=2, d=64, page=16, layout="token", seed=0, extra_rows=0, width=None,
                 q_gain=1.0, row_gap=0, n_pages=None, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        rnd = lambda *s: torch.randn(s, generator=g, device=device)       # noqa: E731
        self.kv, self.new, self.dtype, self.Hq, self.Hkv, self.d, self.page = list(kv), list(new), dtype, Hq, Hkv, d, page
        B = len(kv)
        held = [-(-k // page) for k in kv]
        width = width or max(max(held), 1)
        n_pages = n_pages or sum(held) + 2
        shape = (n_pages, Hkv, page, d) if layout == "head" else (n_pages, page, Hkv, d)
        caches = [torch.full(shape, float("nan"), dtype=DT[dtype], device=device) for _ in range(2)]
        self.k, self.v = (c.permute(0, 2, 1, 3) if layout == "head" else c for c in caches)
        ids = torch.randperm(n_pages, generator=g, device=device)[:sum(held)]
        table = torch.full((B, width), -1, dtype=torch.int32, device=device)
        table[:, ::2] = 1 << 30
        self.K, self.V = [], []                              # what each request's tokens hold, in order
        at = 0
        for b in range(B):
            own = ids[at:at + held[b]]
            at += held[b]
            table[b, :held[b]] = own.to(torch.int32)
            K, V = rnd(kv[b], Hkv, d).to(DT[dtype]), rnd(kv[b], Hkv, d).to(DT[dtype])
            t = torch.arange(kv[b], device=device)
            self.k[own[t // page], t % page] = K
            self.v[own[t // page], t % page] = V
            self.K.append(K)
            self.V.append(V)
        self.table, self.kv_len = table, ints(kv, device)
        self.cu_host = [0] + np.cumsum(new).tolist()
        self.cu = ints(self.cu_host, device)
        rows = sum(new) + extra_rows
        self.q = (rnd(rows, Hq + row_gap, d) * q_gain).to(DT[dtype])[:, :Hq]
        self.max_new = max(max(new), 1)

    def put(self, b, t, K=None, V=None):
        """Other contents of token t of request b."""
        page = self.table[b, t // self.page].long()
        for cache, mine, x in ((self.k, self.K, K), (self.v, self.V, V)):
            if x is not None:
                cache[page, t % self.page] = x
                mine[b][t] = x


def attention(x, scale=None):
    """out, lse in 64 bits, and what a kernel's roundings may amount to: out's tolerance, lse's.  The score of a pair, a sum of d
    products and one scaling, is off by (d + 2) 2^-24 of the sum of its terms' sizes at most, or twice that with the exponent's own
    roundings; the probabilities are rounded once to the storage type, the output once; sums over the keys wander by 2^-24 a term,
    8 standard deviations of which are allowed.  All of it weighs on A = sum of p |v|."""
    scale = x.d ** -0.5 if scale is None else scale
    rows, G, half = x.q.shape[0], x.Hq // x.Hkv, HALF[x.dtype]
    out = torch.full((rows, x.Hq, x.d), float("nan"), dtype=torch.float64, device=x.q.device)
    tol, lse = torch.zeros_like(out), torch.full(out.shape[:2], float("nan"), dtype=torch.float64, device=x.q.device)
    lse_tol = torch.zeros_like(lse)
    for b in range(len(x.kv)):
        r0, n, L = x.cu_host[b], x.new[b], x.kv[b]
        pos = L - n + torch.arange(n, device=x.q.device)
        for c in range(x.Hkv):
            K, V = x.K[b][:, c].double(), x.V[b][:, c].double()
            for h in range(c * G, (c + 1) * G):
                for i0 in range(0, n, 1024):
                    i1 = min(n, i0 + 1024)
                    q = x.q[r0 + i0:r0 + i1, h].double()
                    s = torch.full((i1 - i0, L), -torch.inf, dtype=torch.float64, device=q.device)
                    seen = torch.arange(L, device=q.device)[None, :] <= pos[i0:i1, None]
                    s = torch.where(seen, q @ K.t() * scale, s) if L else s
                    size = torch.where(seen, q.abs() @ K.abs().t() * scale, 0.0).nan_to_num(0, 0, 0).amax(1) if L else q[:, 0] * 0
                    z = torch.logsumexp(s, 1) if L else torch.full_like(size, -torch.inf)
                    p = torch.where(seen, torch.exp(s - z[:, None]), 0.0)
                    # a value that a row does not see does not reach it, whatever it holds
                    Vf = torch.where(torch.isfinite(V), V, 0.0)
                    o, A = p @ Vf, p @ Vf.abs()
                    for t in (~torch.isfinite(V)).any(1).nonzero().flatten().tolist():
                        bad = torch.where(torch.isfinite(V[t]), 0.0, V[t])
                        o = torch.where(seen[:, t:t + 1], o + p[:, t:t + 1] * bad, o)
                    eps = 2 * (x.d + 2) * 2.0 ** -24 * size + 8 * max(L, 64) ** 0.5 * 2.0 ** -24 + 2.0 ** -21
                    sl = slice(r0 + i0, r0 + i1)
                    out[sl, h] = torch.where((pos[i0:i1] >= 0)[:, None], o, torch.zeros_like(o))
                    lse[sl, h] = z
                    tol[sl, h] = half * (o.abs() + (A if x.dtype == "bf16" else 0)) * 1.01 + A * eps[:, None]
                    lse_tol[sl, h] = eps + z.abs().nan_to_num(0, 0, 0) * 2.0 ** -23
    return out, lse, tol, lse_tol


def close(got, ref, tol, what=""):
    """Finite where the reference is, equal where it is infinite, NaN where it is NaN; within tol elsewhere."""
    got = got.double()
    fine = torch.isfinite(ref)
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), f"{what}: NaN elsewhere"
    inf = torch.isinf(ref)
    assert torch.equal(got[inf], ref[inf]), f"{what}: infinities"
    over = ((got - ref).abs() - tol)[fine]
    assert over.numel() == 0 or float(over.max()) <= 0, \
        f"{what}: off by {float((got - ref)[fine].abs().max()):.3e}, {float(over.max()):.3e} over the tolerance"


# ------------------------------------------------------------------ rotary positions
def rotary(d, base=1e6):
    inv = base ** (-np.arange(0, d, 2, dtype=np.float64) / d)
    cut = (d // 8, d // 2 - d // 8)
    return inv, np.repeat(np.arange(3, dtype=np.int32), (cut[0], (cut[1] + 1) // 2, cut[1] // 2))


def cos_sin(positions, inv, axis):
    """[N, d/2] in 64 bits; numpy, positions [axes, N]."""
    angle = positions[np.asarray(axis)].T.astype(np.float64) * inv
    return np.cos(angle), np.sin(angle)


def rotate(x, c, s):
    """x [N, H, d] float64, c and s [N, d/2]"""
    lo, hi = np.split(x, 2, axis=-1)
    c, s = c[:, None], s[:, None]
    return np.concatenate([lo * c - hi * s, hi * c + lo * s], axis=-1)


# ------------------------------------------------------------------ block tables
def update_pages(old, new, table, free, n_free, page, n_rows, offset=None):
    """sparrow_page_update on lists and arrays: (slots, cu, positions, status, table, free, n_free)."""
    table, free = [list(r) for r in table], list(free)
    width, B = len(table[0]), len(old)
    held, need = [-(-o // page) for o in old], [-(-n // page) for n in new]
    none = [-1] * n_rows, [0] * (B + 1), [0] * n_rows
    back = [(b, j) for b in range(B) for j in range(need[b], held[b])]
    take = [(b, j) for b in range(B) for j in range(held[b], need[b])]
    rows = [(b, t) for b in range(B) for t in range(old[b], new[b])]
    status = 0
    if any(not 0 <= x <= width * page for x in list(old) + list(new)):
        status = -2
    elif not 0 <= n_free <= len(free) or n_free + len(back) > len(free):
        status = -3
    elif len(rows) > n_rows:
        status = -1
    elif len(take) > n_free + len(back):
        status = len(take) - n_free - len(back)
    if status:
        return (*none, status, table, free, n_free)
    top = n_free + len(back) - 1
    for k, (b, j) in enumerate(back):
        free[top - k] = table[b][j]
    for k, (b, j) in enumerate(take):
        table[b][j] = free[top - k]
    slots = [table[b][t // page] * page + t % page for b, t in rows] + [-1] * (n_rows - len(rows))
    pos = [t + (offset[b] if offset is not None else 0) for b, t in rows] + [0] * (n_rows - len(rows))
    cu = [0] + np.cumsum([max(n - o, 0) for o, n in zip(old, new)]).tolist()
    return slots, cu, pos, 0, table, free, top + 1 - len(take)
