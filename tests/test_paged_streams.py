"""Calls of the paged operators on a stream of their own (`stream=`): what a call allocates belongs to that stream, whose work alone uses the
memory first, and what it returns is not handed out again before the caller's stream has passed."""
import types

import numpy as np
import pytest
import torch

import paged_ref as ref
from paper_2602_15318_amd import paged

NAMES = ("page_update", "mrope_table", "mrope_append", "chunk_attn")
RETURNED = {"page_update": 4, "mrope_table": 2, "mrope_append": 1, "chunk_attn": 2}


def _args(name, device):
    r = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=device)       # noqa: E731
    i = lambda *x: torch.tensor(x, dtype=torch.int32, device=device)       # noqa: E731
    inv, axis = ref.rotary(64)
    table = torch.arange(80, dtype=torch.int32, device=device).view(2, 40)
    kc, vc = r(80, 16, 2, 64), r(80, 16, 2, 64)
    return {
        "page_update": [i(5, 40), i(20, 30), table, i(7, 8, 9, 10, 11), i(4), 16, 2000],
        "mrope_table": [torch.zeros((3, 3000), dtype=torch.int32, device=device), inv, axis],
        "mrope_append": [r(300, 8, 64), r(300, 2, 64), r(300, 2, 64), torch.zeros((3, 300), dtype=torch.int32, device=device), inv, axis,
                         torch.arange(300, dtype=torch.int32, device=device), kc, vc],
        "chunk_attn": [r(5, 8, 64), kc, vc, table, i(0, 2, 5), i(600, 640), 3],
    }[name]


class Made(torch.Tensor):
    """A tensor that remembers the streams it was recorded on"""


class Gpu:
    """As much of a GPU as the binding asks for, on the CPU: a device that is current or not, its current stream, allocations."""

    def __init__(self, monkeypatch, current_device=0):
        self.device, self.current = current_device, {0: "caller", 1: "other"}
        self.made, self.calls = [], []
        self.dev = torch.device("cuda", 0)
        zeros = torch.zeros

        def empty(*a, **kw):
            kw.pop("device")
            t = zeros(*a, **kw).as_subclass(Made)
            t.on, t.recorded = self.current[0], []
            t.record_stream = t.recorded.append
            self.made.append(t)
            return t

        gpu = self

        class On:
            def __init__(self, stream):
                self.stream = stream

            def __enter__(self):
                self.before = gpu.current[0]
                gpu.current[0] = self.stream.name

            def __exit__(self, *_):
                gpu.current[0] = self.before

        handles = {"caller": 11, "side": 22}
        monkeypatch.setattr(torch, "empty", empty)
        monkeypatch.setattr(torch.cuda, "stream", On)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: self.current[0])
        monkeypatch.setattr(torch.cuda, "current_device", lambda: self.device)
        monkeypatch.setattr(torch.cuda, "set_device", lambda d: setattr(self, "device", getattr(d, "index", d)))
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: handles[self.current[0]], raising=False)
        monkeypatch.setattr(paged, "_tensors", lambda *t: self.dev)
        monkeypatch.setattr(paged, "_native", types.SimpleNamespace(**{n: lambda *a: NotImplemented for n in NAMES}))

        def entry(*a):
            self.calls.append((a[-1], self.device))
            return 0
        monkeypatch.setattr(paged, "lib", types.SimpleNamespace(sparrow_chunk_attn_workspace=lambda *a: 256,
                                                                **{"sparrow_" + n: entry for n in NAMES}))
        self.side = types.SimpleNamespace(name="side", cuda_stream=22, device=self.dev)
        self.own = types.SimpleNamespace(name="caller", cuda_stream=11, device=self.dev)


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("device", [0, 1])
def test_what_a_call_allocates_belongs_to_its_stream(name, device, monkeypatch):
    gpu = Gpu(monkeypatch, device)
    getattr(paged, name)(*_args(name, "cpu"), stream=gpu.side)
    assert gpu.calls == [(22, 0)]
    assert len(gpu.made) >= RETURNED[name] and all(t.on == "side" for t in gpu.made), [t.on for t in gpu.made]
    assert sum(t.recorded == ["caller"] for t in gpu.made) == RETURNED[name]
    assert gpu.current[0] == "caller" and gpu.device == device             # as they were


@pytest.mark.parametrize("name", NAMES)
def test_the_caller_s_own_stream(name, monkeypatch):
    for stream in (None, "own"):
        gpu = Gpu(monkeypatch)
        getattr(paged, name)(*_args(name, "cpu"), stream=stream and gpu.own)
        assert gpu.calls == [(11, 0)] and all(t.on == "caller" and t.recorded == [] for t in gpu.made)


@pytest.mark.parametrize("name", NAMES)
def test_a_stream_of_another_gpu_is_refused(name, monkeypatch):
    gpu = Gpu(monkeypatch)
    far = types.SimpleNamespace(name="far", cuda_stream=33, device=torch.device("cuda", 1))
    with pytest.raises(ValueError, match="stream"):
        getattr(paged, name)(*_args(name, "cpu"), stream=far)
    assert not gpu.calls and gpu.device == 0


def test_an_error_leaves_device_and_stream_as_they_were(monkeypatch):
    gpu = Gpu(monkeypatch, 1)

    def fail(rc):
        raise paged.SparrowError(-1, "no")
    monkeypatch.setattr(paged, "_check", fail)
    for name in NAMES:
        with pytest.raises(paged.SparrowError):
            getattr(paged, name)(*_args(name, "cpu"), stream=gpu.side)
        assert gpu.current[0] == "caller" and gpu.device == 1


def _stream_of(address):
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= address < s["address"] + s["total_size"]:
            return s["stream"]


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_the_allocator_has_them_under_that_stream(name, monkeypatch):
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    side, args, made, real = torch.cuda.Stream(), _args(name, "cuda"), [], torch.empty
    torch.cuda.synchronize()

    def empty(*a, **kw):
        made.append(real(*a, **kw))
        return made[-1]
    monkeypatch.setattr(torch, "empty", empty)
    r = getattr(paged, name)(*args, stream=side)
    torch.cuda.synchronize()
    monkeypatch.setattr(torch, "empty", real)
    assert len(made) >= RETURNED[name] and all(_stream_of(t.data_ptr()) == side.cuda_stream for t in made)
    for t in r if isinstance(r, tuple) else (r,):
        assert any(t is m for m in made)


@pytest.mark.gpu
def test_results_stay_until_the_caller_s_stream_has_passed():
    """A result that the caller's stream still reads, given up: the next call on the side stream gets other memory."""
    side, args = torch.cuda.Stream(), _args("mrope_table", "cuda")
    torch.cuda.synchronize()
    first = paged.mrope_table(*args, stream=side)
    at = {t.data_ptr() for t in first}
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(200_000_000)                           # some tenths of a second of work ahead of the reader
    sums = [t.sum() for t in first]
    behind = torch.cuda.Event()
    behind.record()
    del first
    assert not behind.query()
    second = paged.mrope_table(*args, stream=side)
    assert not at & {t.data_ptr() for t in second}
    torch.cuda.synchronize()
    assert [float(s) for s in sums] == [3000 * 32.0, 0.0]


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_captured_on_a_stream_of_its_own(name):
    """A call on a side stream that a capture has drawn in: replays give what an eager call gives, with eager work in between."""
    args = _args(name, "cuda")
    if name == "chunk_attn":
        for t in args[:3]:
            t.normal_()
    state = [t.clone() if isinstance(t, torch.Tensor) else t for t in args]
    want = getattr(paged, name)(*state)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        got = getattr(paged, name)(*args, stream=side)
        torch.cuda.current_stream().wait_stream(side)
    first = [t.clone() if isinstance(t, torch.Tensor) else t for t in args]
    for _ in range(3):
        for t, x in zip(args, first):
            if isinstance(t, torch.Tensor):
                t.copy_(x)
        for t in got if isinstance(got, tuple) else (got,):
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        for g, w in zip(got if isinstance(got, tuple) else (got,), want if isinstance(want, tuple) else (want,)):
            assert torch.equal(g, w)
        torch.zeros(1 << 20, device="cuda").add_(1)
