"""serve.py's native part against its general code: what it leaves to that code (CPU), that both routes of a call give the same results, of the
same types and shapes, or the same exception (GPU), and whose memory a call on a stream of its own takes (in part on the GPU)."""
import os
import subprocess
import sys
import types

import numpy as np
import pytest
import torch

import paged_ref as ref
import test_paged_streams as streams
from paper_2602_15318_amd import paged, serve
from test_paged_binding_routes import Sub, _flat, _odd_forms

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NAMES = ("mrope_append8", "page_gather", "chunk_attn8", "prefix_attn")
GENERAL = types.SimpleNamespace(**{n: lambda *a: NotImplemented for n in NAMES})
TAIL = {"mrope_append8": (None, None), "page_gather": (None,), "chunk_attn8": (0.0, None, None, True, None, None),
        "prefix_attn": (None, 0.0, None, None, True, None, None)}
MADE = {"mrope_append8": 1, "page_gather": 0, "chunk_attn8": 2, "prefix_attn": 2}


def _calls(device, dtype=torch.bfloat16):
    """name -> arguments of a call that the native part takes"""
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(s, generator=g).to(dtype).to(device)       # noqa: E731
    i = lambda *x: torch.tensor(x, dtype=torch.int32, device=device)       # noqa: E731
    inv, axis = ref.rotary(64)
    table = torch.arange(20, dtype=torch.int32, device=device).view(2, 10)
    k8, v8 = (torch.randn((20, 16, 2, 64), generator=g).to(torch.float8_e4m3fn).to(device) for _ in range(2))
    e = torch.randint(120, 130, (20, 2, 16, 2), generator=g, dtype=torch.uint8).to(device)
    k, v = r(20, 16, 2, 64), r(20, 16, 2, 64)
    return {
        "mrope_append8": [r(4, 8, 64), r(4, 2, 64), r(4, 2, 64), i(*range(12)).view(3, 4), inv, axis, i(3, 90, 17, 50), k8, v8, e],
        "page_gather": [k8, v8, table, i(0, 9, 20), r(20, 2, 64), r(20, 2, 64), e, i(3, 0)],
        "chunk_attn8": [r(5, 8, 64), k8, v8, e, table, i(0, 2, 5), i(100, 147), 3],
        "prefix_attn": [r(5, 8, 64), k, v, table, i(0, 2, 5), i(100, 147), i(0, 2), i(80), 3],
    }


def _variants(name, dtype):
    base = lambda: _calls("cuda", dtype)[name]       # noqa: E731
    z = lambda *s, dt=dtype: torch.zeros(s, dtype=dt, device="cuda")       # noqa: E731
    yield base(), {}
    a = base()
    if name == "mrope_append8":
        x = torch.cat(a[:3], 1)
        yield [x[:, :8], x[:, 8:10], x[:, 10:], *a[3:]], {"q_out": z(4, 8, 64)}
        yield [*a[:3], a[3][0].expand(3, 4), *a[4:7], *(t.transpose(1, 2).contiguous().transpose(1, 2) for t in a[7:9]), a[9]], {}
    elif name == "page_gather":
        k, v = z(2, 20, 64), z(2, 20, 64)
        yield [*a[:4], k.transpose(0, 1), v.transpose(0, 1), a[6], None], {}
        own = _calls("cuda", dtype)["prefix_attn"]
        yield [own[1], own[2], *a[2:6], None, a[7]], {}
    elif name == "chunk_attn8":
        yield a, {"want_lse": False, "scale": 0.25}
        yield a, {"out": z(5, 8, 64), "lse": z(5, 8, dt=torch.float32), "workspace": z(1 << 27, dt=torch.uint8)}
    else:
        yield a, {"want_lse": False, "scale": 0.25}
        yield [*a[:6], None, None, a[8]], {}
        e = _calls("cuda", dtype)["chunk_attn8"]
        yield [a[0], e[1], e[2], *a[3:]], {"exponents": e[3], "out": z(5, 8, 64), "lse": z(5, 8, dt=torch.float32)}
        yield [torch.cat([a[0], a[0]], 1)[:, :8], *a[1:]], {"workspace": z(1 << 28, dt=torch.uint8)}


@pytest.mark.parametrize("name", NAMES)
def test_tensors_on_the_cpu_are_left_to_the_general_code(name):
    assert serve._native.FUNCTIONS, "the native part is not built"
    fn = getattr(serve._native, name)
    args = _calls("cpu")[name]
    assert fn(*args, *TAIL[name]) is NotImplemented
    for what, i, x in _odd_forms(args):
        assert fn(*args[:i], x, *args[i + 1:], *TAIL[name]) is NotImplemented, what
    with pytest.raises(TypeError):
        fn(*args)


def test_a_native_part_that_does_not_fit_is_not_used():
    r = subprocess.run([sys.executable, "-c", """
import sys; sys.modules['paper_2602_15318_amd._native_serve'] = None
import torch
import paper_2602_15318_amd as sp
z = torch.zeros(2, dtype=torch.int32)
c, o = torch.zeros((1, 16, 1, 64)), torch.zeros((1, 1, 64))
try:
    sp.page_gather(c, c, z[:1].view(1, 1), z, o, o)
except ValueError as e:
    print(e)
"""], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    assert "on the GPU" in r.stdout and "RuntimeWarning" in r.stderr and "python -m paper_2602_15318_amd.build" in r.stderr


def _bytes(t):
    return t.contiguous().view(torch.uint8)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("name", NAMES)
def test_both_routes_agree(name, dtype, monkeypatch):
    native, fn, taken, runs = serve._native, getattr(serve, name), [], []

    class Spy:
        def __getattr__(self, n):
            def f(*a):
                r = getattr(native, n)(*a)
                taken.append(r is not NotImplemented)
                return r
            return f

    for part in (Spy(), GENERAL):
        monkeypatch.setattr(serve, "_native", part)
        results = []
        for args, kw in _variants(name, dtype):
            r = fn(*args, **kw)
            torch.cuda.synchronize()
            results.append((type(r), [x if x is None else x.clone() for x in _flat(r) + [a for a in args if isinstance(a, torch.Tensor)]]))
        runs.append(results)
    assert taken and all(taken)
    for (ta, xs), (tb, ys) in zip(*runs):
        assert ta is tb and len(xs) == len(ys)
        for x, y in zip(xs, ys):
            assert (x is None and y is None) or (x.dtype == y.dtype and x.shape == y.shape and torch.equal(_bytes(x), _bytes(y)))
    # refusals: the same exception, or none, by either route
    base = _calls("cuda", dtype)[name]
    with torch.overrides.TorchFunctionMode():
        assert getattr(native, name)(*base, *TAIL[name]) is NotImplemented
    assert getattr(native, name)(*base, *TAIL[name][:-1], torch.cuda.Stream()) is NotImplemented
    bad = [[*base[:i], x, *base[i + 1:]] for _, i, x in _odd_forms(base) if not isinstance(x, (list, np.integer, Sub))]
    bad += [[*base[:i], x.cpu(), *base[i + 1:]] for i, x in enumerate(base) if isinstance(x, torch.Tensor)]
    for args in bad:
        said = []
        for part in (native, GENERAL):
            monkeypatch.setattr(serve, "_native", part)
            try:
                fn(*args)
                said.append(None)
            except (ValueError, TypeError, serve.SparrowError) as e:
                said.append((type(e), str(e)))
        torch.cuda.synchronize()
        assert said[0] == said[1], said


# ------------------------------------------------------------------ streams
def _gpu(monkeypatch, device=0):
    """As much of a GPU as the binding asks for, on the CPU (test_paged_streams.py)"""
    gpu = streams.Gpu(monkeypatch, device)

    def entry(*a):
        gpu.calls.append((a[-1], gpu.device))
        return 0
    monkeypatch.setattr(serve, "_tensors", lambda *t: gpu.dev)
    monkeypatch.setattr(serve, "_native", GENERAL)
    monkeypatch.setattr(serve, "lib", types.SimpleNamespace(sparrow_prefix_attn_workspace=lambda *a: 256, **{"sparrow_" + n: entry for n in NAMES}))
    return gpu


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("device", [0, 1])
def test_what_a_call_allocates_belongs_to_its_stream(name, device, monkeypatch):
    gpu = _gpu(monkeypatch, device)
    getattr(serve, name)(*_calls("cpu")[name], stream=gpu.side)
    assert gpu.calls == [(22, 0)]
    assert len(gpu.made) >= MADE[name] and all(t.on == "side" for t in gpu.made)
    assert sum(t.recorded == ["caller"] for t in gpu.made) == MADE[name]
    assert gpu.current[0] == "caller" and gpu.device == device             # as they were
    gpu = _gpu(monkeypatch)
    far = types.SimpleNamespace(name="far", cuda_stream=33, device=torch.device("cuda", 1))
    with pytest.raises(ValueError, match="stream"):
        getattr(serve, name)(*_calls("cpu")[name], stream=far)
    assert not gpu.calls and gpu.device == 0


def test_two_gpus_are_refused():
    assert serve._tensors is paged._tensors                  # (which test_paged_abi.py holds to it)


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_captured_on_a_stream_of_its_own(name):
    """A call on a side stream that a capture has drawn in: replays give what an eager call gives, with eager work in between."""
    args = _calls("cuda")[name]
    copy = lambda ts: [t.clone() if isinstance(t, torch.Tensor) else t for t in ts]       # noqa: E731
    state = copy(args)
    want = copy(_flat(getattr(serve, name)(*state)))
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    first = copy(args)
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        got = _flat(getattr(serve, name)(*args, stream=side))
        torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        for t, x in zip(args, first):
            if isinstance(t, torch.Tensor):
                t.view(torch.uint8).copy_(x.view(torch.uint8))
        for t in got:
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert torch.equal(g, w)
        torch.zeros(1 << 20, device="cuda").add_(1)
