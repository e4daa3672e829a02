"""sparrow_chunk_attn where scores are large: softmax scales up to the header's limit, and products of millions at ordinary ones.

Queries and keys hold whole numbers whose products stay below 2^24 in sum, so that every score is exact in fp32 and no rounding of it
moves the softmax.  What is left to err: the scale in base 2 (two roundings, a constant's and a product's, 2^-24 each) and the exponent's
own rounding, together 3 2^-24 of a score's distance D from the row's largest, D exp(-D) at most 0.37 of the weight of 1; exp2, the sums and
the division, some 2^-21 each: 2^-19 of A = sum of p |v| in all.  The storage type adds half a step of the output and, in bf16, of each probability.
The log-sum is scaled and converted in four roundings, 2^-22 of it, doubled here, and has the sum's error beside it."""
import math

import numpy as np
import pytest
import torch

import paged_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2602_15318_amd as sp_
    return sp_


def _put_keys(x, keys):
    """Other keys, whole requests at once"""
    for b, K in enumerate(keys):
        t = torch.arange(x.kv[b], device="cuda")
        K = K.to(ref.DT[x.dtype])
        x.k[x.table[b, t // x.page].long(), t % x.page] = K
        x.K[b] = K


def _check(sp, x, scale, what):
    out, lse = sp.chunk_attn(x.q, x.k, x.v, x.table, x.cu, x.kv_len, x.max_new, scale=scale)
    torch.cuda.synchronize()
    real = float(np.float32(scale))
    G, half = x.Hq // x.Hkv, ref.HALF[x.dtype]
    for b in range(len(x.kv)):
        r0, n, L = x.cu_host[b], x.new[b], x.kv[b]
        rows = slice(r0, r0 + n)
        seen = torch.arange(L, device="cuda")[None] <= L - n + torch.arange(n, device="cuda")[:, None]
        for h in range(x.Hq):
            K, V = x.K[b][:, h // G].double(), x.V[b][:, h // G].double()
            raw = torch.where(seen, x.q[rows, h].double() @ K.t(), -torch.inf)
            top = raw.amax(1, keepdim=True)
            p = torch.exp((raw - top) * real)
            z = torch.log(p.sum(1)) + top[:, 0] * real
            p = p / p.sum(1, keepdim=True)
            o, A = p @ V, p @ V.abs()
            ref.close(out[rows, h], o, half * (o.abs() + (A if x.dtype == "bf16" else 0)) * 1.01 + A * 2.0 ** -19, f"{what}, request {b}, head {h}")
            ref.close(lse[rows, h], z, z.abs() * 2.0 ** -21 + 2.0 ** -19, f"{what}, request {b}, head {h}, lse")


# each kernel of the attention: single tokens, chains, chunks
FORMS = [("bf16", 1), ("bf16", 3), ("bf16", 8), ("bf16", 100), ("f32", 1), ("f32", 4), ("f32", 60)]


def _batch(dtype, new, d, seed, width=None):
    kv = [1500, new, new + 1, 700, 64 + new]
    x = ref.Batch(kv, [new] * len(kv), dtype, 14, 2, d, 16, seed=seed, width=width)
    return x, torch.Generator(device="cuda").manual_seed(seed + 1)


def _whole(g, low, high, *shape):
    return torch.randint(low, high + 1, shape, generator=g, device="cuda").float()


@pytest.mark.parametrize("dtype, new", FORMS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("scale", [1e9, 1e12, 1e20, 1e30])
def test_large_scales(sp, dtype, new, d, scale):
    """The largest score takes it all, or those that share its place do."""
    x, g = _batch(dtype, new, d, seed=new)
    x.q = _whole(g, -8, 8, *x.q.shape).to(ref.DT[dtype])
    _put_keys(x, [_whole(g, -8, 8, *K.shape) for K in x.K])
    _check(sp, x, scale, "either sign")
    x.q = _whole(g, 1, 8, *x.q.shape).to(ref.DT[dtype])
    _put_keys(x, [_whole(g, -8, -1, *K.shape) for K in x.K])
    _check(sp, x, scale, "below zero")
    _put_keys(x, [K.abs() for K in x.K])
    _check(sp, x, scale, "above zero")
    _put_keys(x, [torch.where((torch.arange(len(K), device="cuda") % 3 == 0)[:, None, None], 2.0, 1.0).expand(K.shape) for K in x.K])
    _check(sp, x, scale, "many equal")


@pytest.mark.parametrize("dtype, new", FORMS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("offset", [1 << 22, -(1 << 22), 1 << 20, -(1 << 20)])
def test_small_differences_of_large_scores(sp, dtype, new, d, offset):
    """Every second row's scores lie millions from zero and a few units from each other; 2^20 is passed from either side."""
    x, g = _batch(dtype, new, d, seed=new + 1, width=200)
    q = _whole(g, 0, 1, *x.q.shape)
    q[:, :, 0] = 0
    q[::2, :, 0] = 1024
    x.q = q.to(ref.DT[dtype])
    keys = [_whole(g, 0, 1, *K.shape) * (_whole(g, 0, 7, *K.shape[:2], 1) == 0) - (_whole(g, 0, 3, *K.shape) == 0).float() for K in x.K]
    for K in keys:
        K[:, :, 0] = offset // 1024
    _put_keys(x, keys)
    _check(sp, x, math.log(2.0), f"about {offset}, scale ln 2")
    _check(sp, x, 0.0625, f"about {offset}, scale 1/16")


@pytest.mark.parametrize("dtype, new", FORMS)
@pytest.mark.parametrize("d", [64, 128])
def test_scores_that_climb_through_the_range(sp, dtype, new, d):
    """The row's largest score so far grows by factors from one part of the sequence to the next, or falls."""
    x, g = _batch(dtype, new, d, seed=new + 2, width=200)
    x.q = torch.zeros_like(x.q)
    x.q[:, :, 3] = 1.0
    for sign in (1.0, -1.0):
        keys = [torch.zeros(K.shape, device="cuda") for K in x.K]
        for K in keys:
            K[:, :, 3] = sign * 2.0 ** (torch.arange(len(K), device="cuda") // 60).float()[:, None]
        _put_keys(x, keys)
        for scale in (1.0, 1e9, 1e25):
            _check(sp, x, scale, f"{sign} {scale}")


@pytest.mark.parametrize("dtype, new", FORMS)
@pytest.mark.parametrize("d", [64, 128])
def test_one_key_far_below_zero(sp, dtype, new, d):
    x = ref.Batch([new], [new], dtype, 14, 2, d, 16, seed=1)
    x.q = torch.zeros_like(x.q)
    x.q[:, :, 0] = 1.0
    K = torch.zeros_like(x.K[0])
    K[:, :, 0] = -1.0
    _put_keys(x, [K])
    for scale in (1e29, 1e31, 2.0e38):
        out, lse = sp.chunk_attn(x.q, x.k, x.v, x.table, x.cu, x.kv_len, x.max_new, scale=scale)
        torch.cuda.synchronize()
        assert torch.equal(out[0], x.V[0][0].repeat_interleave(7, 0))
        assert ((lse.double() + scale).abs() <= scale * 2.0 ** -21).all()
