"""Refusals of gbs_kv_shared_attention, gbs_kv_attention_mass and gbs_kv_evict, and where their methods take memory; needs no device."""
import ctypes
import types

import pytest
import torch

from paper_2504_13989_b200 import KVCache, binding
from paper_2504_13989_b200 import build as gbs_build
from test_kv_host import ALIGN, BAD_POOLS, INVALID, OK, P, UNSUPPORTED, plan, pool
from test_kv_streams_host import FakeStream, Scene, ints

MOST = binding.GBS_KV_MAX_ITEMS


@pytest.fixture(scope="module")
def lib():
    gbs_build.build()
    return binding.lib()


def shared(lib, pl=None, c=None, seqs=P, cu=P, n=2, t=3, most=2, groups=P, ng=1, own=0, prefix=0, q=P, qt=640, qh=80, heads=8, scale=0.0, flags=1, out=P + 4096, ot=640,
           oh=80, work=P, size=1 << 40):
    return lib.gbs_kv_shared_attention(pl or plan(d=80), ctypes.byref(c or pool()), seqs, cu, n, t, most, groups, ng, own, prefix, q, qt, qh, heads, scale, flags, out, ot,
                                       oh, work, size, None)


def mass(lib, pl=None, c=None, seqs=P, cu=P, n=2, t=3, most=2, q=P, qt=640, qh=80, heads=8, scale=0.0, window=0, flags=1, base=P, decay=1.0, to=P, width=7,
         work=P, size=1 << 40):
    return lib.gbs_kv_attention_mass(pl or plan(d=80), ctypes.byref(c or pool()), seqs, cu, n, t, most, q, qt, qh, heads, scale, window, flags, base, decay, to, width,
                                     work, size, None)


def evict(lib, pl=None, c=None, seqs=P, n=2, keep=9, recent=4, first=5, weights=P, to=P, width=7, kept=P, status=P, work=P, size=1 << 40):
    return lib.gbs_kv_evict(pl or plan(), ctypes.byref(c or pool()), seqs, n, keep, recent, first, weights, to, width, kept, status, work, size, None)


@pytest.mark.parametrize("f", [shared, mass, evict])
def test_pools_plans_and_nothing_to_do(lib, f):
    more = {} if f is evict else {"t": 0}
    assert f(lib, n=0, **more) == OK
    for change, want in BAD_POOLS:
        assert f(lib, c=pool(**change)) == want
    assert f(lib, pl=plan(bits=3)) == UNSUPPORTED and f(lib, pl=plan(d=100)) == UNSUPPORTED
    for n in (-1, MOST + 1):
        assert f(lib, n=n) == INVALID
    assert f(lib, seqs=None, n=6) == INVALID and f(lib, seqs=P + 1) == ALIGN


def test_shared_attention(lib):
    f = lambda **kw: shared(lib, **kw)  # noqa: E731
    assert f(ng=0) == INVALID and f(ng=MOST + 1) == INVALID and f(groups=None, ng=2) == INVALID and f(groups=P + 2) == ALIGN and f(own=-1) == INVALID and f(prefix=-1) == INVALID
    assert f(heads=6) == INVALID and f(heads=0) == INVALID and f(most=0) == INVALID and f(cu=None, n=3, most=2) == INVALID and f(cu=None) == INVALID
    assert f(most=1 << 30) == INVALID and f(t=-1) == INVALID and f(t=1 << 29) == INVALID and f(flags=2) == INVALID
    assert f(scale=float("inf")) == INVALID and f(scale=float("nan")) == INVALID
    assert f(q=None) == INVALID and f(out=None) == INVALID and f(work=None) == INVALID and f(size=0) == INVALID and f(out=P) == INVALID
    assert f(qt=72) == INVALID and f(oh=72) == INVALID and f(qt=641) == ALIGN and f(oh=84) == ALIGN
    assert f(q=P + 8) == ALIGN and f(out=P + 4) == ALIGN and f(work=P + 8) == ALIGN and f(cu=P + 2) == ALIGN
    assert f(t=0, q=None) == OK and f(n=0, q=None) == OK
    size, r = ctypes.c_int64(-1), ctypes.byref(pool())
    w = lib.gbs_kv_shared_attention_workspace
    for prefix in (0, 1 << 30):                                # whatever the call judges of sharing
        assert w(plan(d=80), r, 2, 3, 2, 1, prefix, 8, ctypes.byref(size)) == OK and size.value > 0
        assert f(size=size.value - 1, prefix=prefix) == INVALID
    for bad in ((-1, 3, 2, 1, 0, 8), (2, -1, 2, 1, 0, 8), (2, 3, 0, 1, 0, 8), (2, 3, 2, 0, 0, 8), (2, 3, 2, MOST + 1, 0, 8), (2, 3, 2, 1, 0, 6), (2, 1 << 40, 2, 1, 0, 8),
                (2, 3, 2, 1, -1, 8)):
        assert w(plan(d=80), r, *bad, ctypes.byref(size)) == INVALID
    assert w(plan(d=80), r, 2, 3, 2, 1, 0, 8, None) == INVALID


def test_attention_mass(lib):
    f = lambda **kw: mass(lib, **kw)  # noqa: E731
    assert f(width=0) == INVALID and f(decay=float("nan")) == INVALID and f(decay=float("inf")) == INVALID and f(base=None) == INVALID
    assert f(to=None) == INVALID and f(to=P + 2) == ALIGN and f(base=P + 2) == ALIGN
    assert f(heads=6) == INVALID and f(most=0) == INVALID and f(cu=None) == INVALID and f(t=1 << 29) == INVALID and f(window=-1) == INVALID and f(flags=2) == INVALID
    assert f(q=None) == INVALID and f(work=None) == INVALID and f(size=0) == INVALID and f(qt=72) == INVALID and f(qt=641) == ALIGN and f(q=P + 8) == ALIGN
    assert f(t=0, q=None) == OK and f(n=0, to=None) == OK
    size, r = ctypes.c_int64(-1), ctypes.byref(pool())
    w = lib.gbs_kv_attention_mass_workspace
    assert w(plan(d=80), r, 2, 3, 2, 8, 7, ctypes.byref(size)) == OK and f(size=size.value - 1) == INVALID
    for bad in ((-1, 3, 2, 8, 7), (2, -1, 2, 8, 7), (2, 3, 0, 8, 7), (2, 3, 2, 6, 7), (2, 3, 2, 8, 0)):
        assert w(plan(d=80), r, *bad, ctypes.byref(size)) == INVALID
    assert w(plan(d=80), r, 2, 3, 2, 8, 7, None) == INVALID
    for width in (1 << 20, 1 << 40, (1 << 63) - 1):                                # scores have room up to a limit
        assert w(plan(d=80), r, 2, 3, 2, 8, width, ctypes.byref(size)) == OK and 0 < size.value < 300 << 20


def test_evict(lib):
    f = lambda **kw: evict(lib, **kw)  # noqa: E731
    assert f(keep=0, recent=0, first=0) == INVALID and f(recent=-1) == INVALID and f(first=-1) == INVALID and f(recent=5) == INVALID
    assert f(recent=2 ** 31 - 1, first=2 ** 31 - 1) == INVALID and f(width=0) == INVALID
    for name in ("weights", "to", "kept", "status", "work"):
        assert f(**{name: None}) == INVALID and f(**{name: P + 2}) == ALIGN
    size, r = ctypes.c_int64(-1), ctypes.byref(pool())
    w = lib.gbs_kv_evict_workspace
    assert w(plan(), r, 2, 2 ** 31 - 1, ctypes.byref(size)) == OK and size.value < 1 << 16               # no more than a sequence can have
    assert w(plan(), r, 2, 17, ctypes.byref(size)) == OK and size.value > 0 and f(keep=17, size=size.value - 1) == INVALID
    assert w(plan(), r, -1, 17, ctypes.byref(size)) == INVALID and w(plan(), r, 2, 0, ctypes.byref(size)) == INVALID and w(plan(), r, 2, 17, None) == INVALID


x = torch.zeros(3, 2, 128, dtype=torch.bfloat16)
m, b = torch.zeros(3, 2, 9), torch.zeros(3, 2, 9)
s, cu, cuts = ints(0, 1, 2), ints(0, 1, 2, 3), ints(0, 3)
CALLS = [  # name, arguments, of which tensors, which of the results are new
    ("shared_attention", dict(q=x, seqs=s, cu_tokens=cu, groups=cuts), (x, s, cu, cuts), 1),
    ("attention_mass", dict(q=x, mass=m, seqs=s, cu_tokens=cu, base=b), (x, m, b, s, cu), 0),
    ("evict", dict(mass=m, keep=4, seqs=s, into=b), (m, b, s), 2),
]


@pytest.mark.parametrize("name,kw,tensors,results", CALLS)
def test_memory_comes_from_the_stream_of_the_call(name, kw, tensors, results, monkeypatch):
    a = Scene(monkeypatch)
    a.cache.page_table = torch.zeros(3, 2, dtype=torch.int32)
    got = binding._PYTHON_KV_METHODS[name](a.cache, stream=a.side, **kw)
    assert [where for _, where in a.empty] == [a.side] * (results + 1)
    for g in (got if isinstance(got, tuple) else (got,))[:results]:
        assert (g.data_ptr(), a.current) in a.recorded
    for i in tensors + a.cache._kept:
        assert (i.data_ptr(), a.side) in a.recorded
    a = Scene(monkeypatch)
    binding._PYTHON_KV_METHODS[name](a.cache, **kw)
    assert not a.recorded
    with pytest.raises(ValueError):
        binding._PYTHON_KV_METHODS[name](a.cache, stream=FakeStream("far", 1), **kw)


def cache_of():
    c = object.__new__(KVCache)
    c.plan = types.SimpleNamespace(handle=1, info=types.SimpleNamespace(d=128, asymmetric=0))
    c.n_kv_heads, c.page_size, c.pages, c.page_table = 2, 16, torch.zeros(4, 4352, dtype=torch.uint8), torch.zeros(3, 2, dtype=torch.int32)
    return c


def test_the_methods_refuse_what_the_library_cannot_see(monkeypatch):
    monkeypatch.setattr(binding, "_check_buffer", lambda *a: None)
    monkeypatch.setattr(KVCache, "_rows", lambda *a: None)
    c, f = cache_of(), binding._PYTHON_KV_METHODS
    for bad in (torch.zeros(2, 2, 9), torch.zeros(3, 1, 9), torch.zeros(3, 2), torch.zeros(3, 2, 9, 1)):
        with pytest.raises(ValueError):
            f["attention_mass"](c, x, bad)
        with pytest.raises(ValueError):
            f["evict"](c, bad, 4)
    with pytest.raises(ValueError):
        f["attention_mass"](c, x, m, base=torch.zeros(3, 2, 8))
    with pytest.raises(ValueError):
        f["evict"](c, m, 4, into=torch.zeros(3, 2, 8))
    for kw in (dict(keep=2 ** 32 + 4), dict(keep=4, recent=2 ** 32), dict(keep=4, first=2 ** 40)):
        with pytest.raises(ValueError):
            f["evict"](c, m, **kw)
    for bad in (ints(0), torch.zeros(2, 2, dtype=torch.int32)):
        with pytest.raises(ValueError):
            f["shared_attention"](c, x, groups=bad)
    with pytest.raises(ValueError):
        f["shared_attention"](c, x[0])
    with pytest.raises(ValueError):
        f["shared_attention"](c, x, max_own=2 ** 32)
    with pytest.raises(ValueError):
        f["shared_attention"](c, x, max_prefix=2 ** 32)
