"""The serving operators as a program runs them: a video prefilled once into an 8-bit cache, questions about it that share its pages, answered
token by token, drafts verified as a tree over what is read back; every length on the GPU, a step captured and replayed."""
import numpy as np
import pytest
import torch

import paged_ref as ref
import serve_ref as s8

pytestmark = pytest.mark.gpu
# Weights and outputs are rounded to bf16 once each, half a step 2^-8: 2^-8 (A + |o|), with A = sum of p |v| <= 2 for these values, N(0, 1) and quantised;
# a query that falls the other way there shifts scores by 2^-8 of some units.  The sum stays below this.
TOL = 2e-2


@pytest.fixture(scope="module")
def sp():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2602_15318_amd as sp_
    return sp_


class Server:
    """One video of `video` tokens on shared pages, B questions about it behind them on pages of their own."""

    def __init__(self, sp, B, Hq, Hkv, d, page, video, room):
        self.sp, self.B, self.Hq, self.Hkv, self.d, self.page, self.video = sp, B, Hq, Hkv, d, page, video
        shared, own = video // page, room // page
        n = shared + B * own
        self.kc, self.vc = (torch.full((n, page, Hkv, d), 0x7f, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
        self.exps = torch.full((n, Hkv, page, 2), 255, dtype=torch.uint8, device="cuda")
        ids = torch.randperm(n, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(torch.int32)
        self.table = torch.cat([ids[:shared].expand(B, shared), ids[shared:].view(B, own), ids.new_full((B, s8.wide_table(B, Hkv, d, page)), -1)],
                               1).contiguous()                    # room for long contexts, so that the video is read once
        self.len = torch.full((B,), video, dtype=torch.int32, device="cuda")
        self.inv, self.axis = ref.rotary(d)
        self.start, self.prefix = ref.ints([0, B]), ref.ints([video])

    def slots(self, b, first, n):
        t = torch.arange(n, device="cuda") + first
        return (self.table[b, t // self.page] * self.page + t % self.page).to(torch.int32)

    def write(self, qkv, slots, pos):
        q, k, v = qkv[:, :self.Hq], qkv[:, self.Hq:self.Hq + self.Hkv], qkv[:, self.Hq + self.Hkv:]
        return self.sp.mrope_append8(q, k, v, pos.expand(3, -1), self.inv, self.axis, slots, self.kc, self.vc, self.exps)

    def step(self, qkv, out, lse):
        """One token of every request: written behind its context, attended with the shared prefix."""
        t = self.len.long()
        slots = (self.table.gather(1, (t // self.page)[:, None])[:, 0] * self.page + t % self.page).to(torch.int32)
        q = self.write(qkv, slots, self.len)
        self.len += 1
        return self.sp.prefix_attn(q, self.kc, self.vc, self.table, self.cu, self.len, self.start, self.prefix, 1, exponents=self.exps, out=out, lse=lse)


def _held(s, b, n):
    """What the cache holds of request b: K, V [n, Hkv, d]"""
    out = [torch.empty((n, s.Hkv, s.d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    return s.sp.page_gather(s.kc, s.vc, s.table[b:b + 1], ref.ints([0, n]), *out, exponents=s.exps)


def _plain(q, K, V, pos):
    G = q.shape[1] // K.shape[1]
    sc = torch.einsum("nhd,mhd->hnm", q.double().cpu(), K.double().cpu().repeat_interleave(G, 1)) * q.shape[2] ** -0.5
    sc = sc.masked_fill(torch.arange(K.shape[0])[None] > pos[:, None], -torch.inf)
    return torch.einsum("hnm,mhd->nhd", torch.softmax(sc, -1), V.double().cpu().repeat_interleave(G, 1))


def _filled(sp, B=3, Hq=8, Hkv=2, d=128, page=16, video=320):
    s = Server(sp, B, Hq, Hkv, d, page, video, 128)
    g = torch.Generator(device="cuda").manual_seed(5)
    rows = lambda n: torch.randn((n, Hq + 2 * Hkv, d), generator=g, device="cuda").bfloat16()       # noqa: E731
    x = rows(video)
    for a in range(0, video, 100):                           # the video, 100 tokens at a time
        n = min(100, video - a)
        pos = torch.arange(a, a + n, dtype=torch.int32, device="cuda")
        q = s.write(x[a:a + n], s.slots(0, a, n), pos)
        out, _ = sp.chunk_attn8(q, s.kc, s.vc, s.exps, s.table[:1], ref.ints([0, n]), ref.ints([a + n]), n)
        K, V = _held(s, 0, a + n)
        assert (out.double().cpu() - _plain(q, K, V, torch.arange(a, a + n))).abs().max() < TOL
    n = [7, 30, 12][:B]                                      # the questions, all at once
    qs, slots = rows(sum(n)), torch.cat([s.slots(b, video, m) for b, m in enumerate(n)])
    pos = torch.cat([torch.arange(video, video + m, dtype=torch.int32) for m in n]).cuda()
    q = s.write(qs, slots, pos)
    cu = [0] + np.cumsum(n).tolist()
    s.len = ref.ints([video + m for m in n])
    out, _ = sp.prefix_attn(q, s.kc, s.vc, s.table, ref.ints(cu), s.len, s.start, s.prefix, max(n), exponents=s.exps)
    for b, m in enumerate(n):
        K, V = _held(s, b, video + m)
        want = _plain(q[cu[b]:cu[b + 1]], K, V, torch.arange(video, video + m))
        assert (out[cu[b]:cu[b + 1]].double().cpu() - want).abs().max() < TOL
    s.cu = ref.ints(range(B + 1))
    return s, rows


def test_a_video_questions_and_answers(sp):
    s, rows = _filled(sp)
    out, lse = torch.empty((s.B, s.Hq, s.d), dtype=torch.bfloat16, device="cuda"), torch.empty((s.B, s.Hq), device="cuda")
    for _ in range(5):
        x = rows(s.B)
        before = s.len.tolist()
        s.step(x, out, lse)
        for b, t in enumerate(before):                       # the token's query once more, over what the cache holds
            K, V = _held(s, b, t + 1)
            c, sn = ref.cos_sin(np.full((3, 1), t), s.inv, s.axis)
            q = torch.from_numpy(ref.rotate(x[b:b + 1, :s.Hq].double().cpu().numpy(), c, sn)).bfloat16()
            assert (out[b:b + 1].double().cpu() - _plain(q, K, V, torch.tensor([t]))).abs().max() < TOL


def test_a_tree_of_drafts_over_what_is_read_back(sp):
    """page_gather lays the contexts out for sparrow_verify_attn, which takes draft trees."""
    s, rows = _filled(sp)
    L, n_q = s.len.tolist(), 5
    parent = np.array([-1, 0, 0, 1, 2], np.int32)
    total = sum(L) + s.B * n_q
    k, v = (torch.zeros((s.Hkv, total, s.d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cu, at = [0], 0
    for n in L:
        at += n + n_q
        cu.append(at)
    for b in range(s.B):                                     # each context where its sequence begins
        sp.page_gather(s.kc, s.vc, s.table[b:b + 1], ref.ints([0, L[b]]), k.permute(1, 0, 2)[cu[b]:cu[b] + L[b]], v.permute(1, 0, 2)[cu[b]:cu[b] + L[b]],
                       exponents=s.exps)
    drafts = rows(s.B * n_q)
    for b in range(s.B):
        for t, w in ((k, 0), (v, 1)):
            t[:, cu[b] + L[b]:cu[b + 1]] = drafts[b * n_q:(b + 1) * n_q, s.Hq + w * s.Hkv:s.Hq + (w + 1) * s.Hkv].transpose(0, 1)
    q = drafts[:, :s.Hq].contiguous()
    out, _ = sp.verify_attn(q, k.permute(1, 0, 2), v.permute(1, 0, 2), np.array(cu, np.int32), torch.from_numpy(parent).cuda(), n_q)
    seen = np.zeros((n_q, n_q), bool)
    for i in range(n_q):
        j = i
        while j >= 0:
            seen[i, j] = True
            j = parent[j]
    for b in range(s.B):
        K, V = k[:, cu[b]:cu[b + 1]].double().cpu(), v[:, cu[b]:cu[b + 1]].double().cpu()
        G = s.Hq // s.Hkv
        sc = torch.einsum("nhd,hmd->hnm", q[b * n_q:(b + 1) * n_q].double().cpu(), K.repeat_interleave(G, 0)) * s.d ** -0.5
        mask = torch.cat([torch.ones(n_q, L[b], dtype=torch.bool), torch.from_numpy(seen)], 1)
        want = torch.einsum("hnm,hmd->nhd", torch.softmax(sc.masked_fill(~mask, -torch.inf), -1), V.repeat_interleave(G, 0))
        assert (out[b * n_q:(b + 1) * n_q].double().cpu() - want).abs().max() < TOL


def test_a_captured_step(sp):
    """The step in a graph, replayed as the requests grow, against eager steps on a twin; eager work in between."""
    a, rows = _filled(sp)
    b, _ = _filled(sp)
    x = [rows(a.B) for _ in range(20)]
    qkv = x[0].clone()
    out, lse = torch.empty((a.B, a.Hq, a.d), dtype=torch.bfloat16, device="cuda"), torch.empty((a.B, a.Hq), device="cuda")
    out_b, lse_b = torch.empty_like(out), torch.empty_like(lse)
    state = lambda s: [s.kc.view(torch.uint8), s.vc.view(torch.uint8), s.exps, s.len]       # noqa: E731
    keep = [t.clone() for t in state(a)]
    a.step(qkv, out, lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step(qkv, out, lse)
    for t, old in zip(state(a), keep):
        t.copy_(old)
    for step in range(20):
        qkv.copy_(x[step])
        graph.replay()
        torch.cuda.synchronize()
        b.step(x[step], out_b, lse_b)
        assert torch.equal(out, out_b) and torch.equal(lse, lse_b), step
        for t, u in zip(state(a), state(b)):
            assert torch.equal(t, u), step
        torch.zeros(1 << 20, device="cuda").add_(1)


def test_two_graphs_that_share_a_workspace(sp):
    """Replayed one after the other on one stream, in any order."""
    s, rows = _filled(sp)
    q = [rows(s.B)[:, :s.Hq].contiguous() for _ in range(2)]
    args = lambda i: (q[i], s.kc, s.vc, s.table, s.cu, s.len, s.start, s.prefix, 1)       # noqa: E731
    want = [sp.prefix_attn(*args(i), exponents=s.exps)[0].clone() for i in range(2)]
    ws = torch.empty((sp.prefix_attn_workspace_bytes(q[0], s.kc, s.vc, s.B, 1, 1, exponents=s.exps),), dtype=torch.uint8, device="cuda")
    outs, graphs = [torch.empty_like(w) for w in want], []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            sp.prefix_attn(*args(i), exponents=s.exps, out=outs[i], workspace=ws, want_lse=False)
        graphs.append(g)
    for i in (0, 1, 1, 0, 0, 1):
        outs[i].fill_(9)
        graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[i], want[i])
