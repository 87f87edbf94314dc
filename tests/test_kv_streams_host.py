"""Where KVCache's calls take their memory when they are given a stream; needs no device: streams, the allocator and the library are stand-ins."""
import contextlib
import types

import pytest
import torch

from paper_2504_13989_b200 import KVCache, binding


class FakeStream:
    def __init__(self, name, index=0):
        self.name, self.cuda_stream, self.device = name, 7, types.SimpleNamespace(index=index)

    def __repr__(self):
        return self.name


class Scene:
    """A KVCache over CPU tensors whose library answers 0 to everything, and notes of who allocated and recorded what."""

    def __init__(self, monkeypatch):
        self.current, self.side = FakeStream("current"), FakeStream("side")
        self.now, self.empty, self.recorded, self.calls = self.current, [], [], []
        real = torch.empty

        @contextlib.contextmanager
        def stream(s):
            was, self.now = self.now, s
            yield
            self.now = was

        def empty(*a, **kw):
            t = real(*a, **{k: v for k, v in kw.items() if k != "device"})
            self.empty.append((t.data_ptr(), self.now))
            return t
        monkeypatch.setattr(torch.cuda, "stream", stream)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: self.now)
        monkeypatch.setattr(torch, "empty", empty)
        monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: self.recorded.append((t.data_ptr(), s)))
        scene = self

        class Library:
            def __getattr__(self, name):
                def call(*a):
                    if name == "gbs_kv_attention_workspace":
                        a[-1]._obj.value = 4096
                    scene.calls.append((name, a))
                    return 0
                return call
        monkeypatch.setattr(binding, "lib", lambda: Library())
        monkeypatch.setattr(binding, "_check_buffer", lambda *a: None)
        monkeypatch.setattr(KVCache, "_rows", lambda *a: None)
        c = object.__new__(KVCache)
        c.plan = types.SimpleNamespace(handle=1, info=types.SimpleNamespace(d=128, asymmetric=0))
        c.n_kv_heads, c.page_size = 2, 16

        class Pages(torch.Tensor):                              # a CPU tensor that says it is on the streams' device
            device = self.side.device
        c.pages = torch.zeros(4, 4352, dtype=torch.uint8).as_subclass(Pages)
        c.page_table = torch.zeros(3, 2, dtype=torch.int32)
        c._kept = (c.page_table,)
        c._c = binding.KVCacheStruct()
        self.cache = c


def ints(*v):
    return torch.tensor(v, dtype=torch.int32)


x = torch.zeros(3, 2, 128, dtype=torch.bfloat16)
s, t, cu, page_map = ints(0, 1, 2), ints(1, 1, 1), ints(0, 1, 2, 3), ints(0, 0, 0, 0)
CALLS = [  # name, arguments, of which tensors, how many results, whether there is memory that no result is
    ("extend", dict(seqs=s, counts=t), (s, t), 1, 0), ("fork", dict(src=s, dst=t), (s, t), 1, 0), ("free", dict(seqs=s), (s,), 0, 0),
    ("compact", dict(), (), 1, 1), ("compact", dict(page_map=page_map), (page_map,), 1, 0),
    ("append", dict(k=x, v=x, seqs=s, cu_tokens=cu, status=t), (x, s, cu, t), 0, 0), ("read", dict(seqs=s, cu_tokens=cu, n_tokens=3), (s, cu), 2, 0),
    ("attention", dict(q=x, seqs=s, cu_tokens=cu), (x, s, cu), 1, 1),
]


@pytest.mark.parametrize("name,kw,tensors,results,hidden", CALLS)
def test_memory_comes_from_the_stream_of_the_call(name, kw, tensors, results, hidden, monkeypatch):
    a = Scene(monkeypatch)
    if name == "compact":
        kw = dict(kw, into=a.cache)
    got = binding._PYTHON_KV_METHODS[name](a.cache, stream=a.side, **kw)
    assert [where for _, where in a.empty] == [a.side] * (results + hidden)
    got = () if got is None else got if isinstance(got, tuple) else (got,)
    for g in got:                                              # the caller's stream goes on with these
        assert (g.data_ptr(), a.current) in a.recorded
    for i in tensors + a.cache._kept:                          # the caller may let go of these at once
        assert (i.data_ptr(), a.side) in a.recorded
    assert a.calls[-1][0] == "gbs_kv_" + name + "_extended" * (name == "append") and a.side.cuda_stream in a.calls[-1][1]


@pytest.mark.parametrize("name,kw,tensors,results,hidden", CALLS)
def test_without_a_stream_nothing_is_recorded(name, kw, tensors, results, hidden, monkeypatch):
    a = Scene(monkeypatch)
    if name == "compact":
        kw = dict(kw, into=a.cache)
    binding._PYTHON_KV_METHODS[name](a.cache, **kw)
    assert [where for _, where in a.empty] == [a.current] * (results + hidden) and not a.recorded


def test_a_stream_of_another_device_is_refused(monkeypatch):
    a = Scene(monkeypatch)
    with pytest.raises(ValueError):
        binding._PYTHON_KV_METHODS["free"](a.cache, s, stream=FakeStream("far", 1))
    assert not a.calls
