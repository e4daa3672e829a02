"""paged.py's native part against its general code: what it leaves to that code (CPU), and that both routes of a call give the same
results, of the same types and shapes, or the same exception (GPU)."""
import os
import subprocess
import sys
import types

import numpy as np
import pytest
import torch

import paged_ref as ref
from paper_2602_15318_amd import paged

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NAMES = ("page_update", "mrope_table", "mrope_append", "chunk_attn")
GENERAL = types.SimpleNamespace(**{n: lambda *a: NotImplemented for n in NAMES})


class Sub(torch.Tensor):
    pass


def _calls(device, dtype=torch.bfloat16):
    """name -> (arguments of a call that the native part takes, names of those changed in place)"""
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(s, generator=g).to(dtype).to(device)       # noqa: E731
    i = lambda *x: torch.tensor(x, dtype=torch.int32, device=device)       # noqa: E731
    inv, axis = ref.rotary(64)
    table = torch.arange(6, dtype=torch.int32, device=device).view(2, 3)
    kc, vc = r(6, 16, 2, 64), r(6, 16, 2, 64)
    return {
        "page_update": [i(5, 40), i(20, 30), table, i(7, 8, 9, 10, 11), i(4), 16, 20],
        "mrope_table": [i(*range(12)).view(3, 4), inv, axis],
        "mrope_append": [r(4, 8, 64), r(4, 2, 64), r(4, 2, 64), i(*range(12)).view(3, 4), inv, axis, i(3, 90, 17, 50), kc, vc],
        "chunk_attn": [r(5, 8, 64), kc, vc, table, i(0, 2, 5), i(30, 47), 3],
    }


TAIL = {"page_update": (None, None, None), "mrope_table": (None, None, None), "mrope_append": (None, None),
        "chunk_attn": (0.0, None, None, True, None, None)}


def _odd_forms(args):
    """(what, index, other value) of forms that the general code converts or refuses, one argument at a time"""
    for i, a in enumerate(args):
        if isinstance(a, np.ndarray):
            yield f"{i} list", i, a.tolist()
            yield f"{i} other type", i, a.astype(np.float32 if a.dtype == np.float64 else np.int64)
            yield f"{i} every other", i, np.repeat(a, 2)[::2]
            yield f"{i} short", i, a[:-1]
        elif isinstance(a, torch.Tensor):
            yield f"{i} subclass", i, a.as_subclass(Sub)
            yield f"{i} float64", i, a.double()
            if a.numel() > 1:
                yield f"{i} with gaps", i, torch.stack([a, a], -1)[..., 0]
        else:
            yield f"{i} numpy", i, np.int64(a)


@pytest.mark.parametrize("name", NAMES)
def test_tensors_on_the_cpu_are_left_to_the_general_code(name):
    assert paged._native.FUNCTIONS, "the native part is not built"
    fn = getattr(paged._native, name)
    args = _calls("cpu")[name]
    assert fn(*args, *TAIL[name]) is NotImplemented
    for what, i, x in _odd_forms(args):
        assert fn(*args[:i], x, *args[i + 1:], *TAIL[name]) is NotImplemented, what
    with pytest.raises(TypeError):
        fn(*args)


def test_a_native_part_that_does_not_fit_is_not_used():
    r = subprocess.run([sys.executable, "-c", """
import sys; sys.modules['paper_2602_15318_amd._native_paged'] = None
import torch
import paper_2602_15318_amd as sp
z = torch.zeros(2, dtype=torch.int32)
try:
    sp.page_update(z, z, z.view(2, 1), z, z[:1], 16, 0)
except ValueError as e:
    print(e)
"""], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    assert "on the GPU" in r.stdout and "RuntimeWarning" in r.stderr and "python -m paper_2602_15318_amd.build" in r.stderr


def _flat(r):
    return list(r) if isinstance(r, tuple) else [r]


def _variants(name, dtype):
    base = lambda: _calls("cuda", dtype)[name]       # noqa: E731
    e = lambda *s, dt=torch.int32: torch.zeros(s, dtype=dt, device="cuda")       # noqa: E731
    yield base(), {}
    if name == "page_update":
        yield base(), {"pos_offset": torch.tensor([3, -4], dtype=torch.int32, device="cuda")}
        yield base(), {"outputs": (e(20), e(3), e(20), e(1))}
    elif name == "mrope_table":
        yield [torch.arange(4, dtype=torch.int32, device="cuda"), *base()[1:2], 0 * base()[2]], {}
        yield base(), {"cos": e(4, 32, dt=torch.float32)}
    elif name == "mrope_append":
        a = base()
        x = torch.cat(a[:3], 1)
        yield [x[:, :8], x[:, 8:10], x[:, 10:], *a[3:]], {"q_out": e(4, 8, 64, dt=dtype)}
        yield [a[0], a[1], a[2], a[3][0].expand(3, 4), *a[4:7], a[7].transpose(1, 2).contiguous().transpose(1, 2),
               a[8].transpose(1, 2).contiguous().transpose(1, 2)], {}
    else:
        a = base()
        yield a, {"want_lse": False, "scale": 0.25}
        yield a, {"out": e(5, 8, 64, dt=dtype), "lse": e(5, 8, dt=torch.float32), "workspace": e(1 << 24, dt=torch.uint8)}
        yield [torch.cat([a[0], a[0]], 1)[:, :8], *a[1:]], {}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("name", NAMES)
def test_both_routes_agree(name, dtype, monkeypatch):
    native = paged._native
    fn = getattr(paged, name)
    taken = []

    class Spy:
        def __getattr__(self, n):
            def f(*a):
                r = getattr(native, n)(*a)
                taken.append(r is not NotImplemented)
                return r
            return f

    runs = []
    for part in (Spy(), GENERAL):
        monkeypatch.setattr(paged, "_native", part)
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
            assert (x is None and y is None) or (x.dtype == y.dtype and x.shape == y.shape and torch.equal(x, y))
    # refusals: the same exception, or none, by either route
    base = _calls("cuda", dtype)[name]
    with torch.overrides.TorchFunctionMode():
        assert getattr(native, name)(*base, *TAIL[name]) is NotImplemented
    assert getattr(native, name)(*base, *TAIL[name][:-1], torch.cuda.Stream()) is NotImplemented
    bad = [[*base[:i], x, *base[i + 1:]] for _, i, x in _odd_forms(base) if not isinstance(x, (list, np.integer, Sub))]
    bad += [[*base[:i], x.cpu(), *base[i + 1:]] for i, x in enumerate(base) if isinstance(x, torch.Tensor)]
    if name == "page_update":
        bad.append([*base[:5], 24, 20])                  # the library's own refusal
    for args in bad:
        said = []
        for part in (native, GENERAL):
            monkeypatch.setattr(paged, "_native", part)
            try:
                fn(*args)
                said.append(None)
            except (ValueError, TypeError, paged.SparrowError) as e:
                said.append((type(e), str(e)))
        torch.cuda.synchronize()
        assert said[0] == said[1], said
