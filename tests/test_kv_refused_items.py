"""Items that gbs_kv_extend refused: gbs_kv_append_extended leaves their rows out, in a captured step too."""
import ctypes
import inspect

import pytest
import torch

import kv_util
from paper_2504_13989_b200 import KVCache, Plan, binding
from paper_2504_13989_b200 import build as gbs_build
from test_kv_host import ALIGN, INVALID, OK, P, plan, pool

DEV = kv_util.DEV


@pytest.fixture(scope="module", autouse=True)
def built():
    gbs_build.build()


def test_refusals():
    lib, c = binding.lib(), pool()
    a = lambda n=2, t=3, k=P, cu=P, status=P: lib.gbs_kv_append_extended(plan(), ctypes.byref(c), P, cu, n, t, k, P, 512, 128, status, None)  # noqa: E731
    assert a(status=P + 2) == ALIGN and a(status=P + 1) == ALIGN and a(k=None) == INVALID and a(cu=None) == INVALID and a(n=-1) == INVALID
    assert a(n=0) == OK and a(t=0) == OK and a(n=0, status=None) == OK


def test_the_binding_names_it_last():
    """Positional calls of the older form stay what they were."""
    assert list(inspect.signature(KVCache.append).parameters) == ["self", "k", "v", "seqs", "cu_tokens", "stream", "status"]


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def held(cache, seq):
    """What a sequence's pages hold: its tokens' codes and scales."""
    return [t.clone() for t in kv_util.rows_of(cache, seq)]


@pytest.mark.gpu
@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("asym", [False, True])
def test_a_step_that_runs_out_of_pages_beside_a_fork(captured, asym):
    """Sequence 1 shares the full pages of sequence 0; when there is no page left, neither loses a token."""
    with Plan(128, 128, 1, 4, 128, 0.9, asymmetric=asym) as plan:
        cache = KVCache.create(plan, 5, 2, 16, 3, 4, DEV)
        gen = torch.Generator(device=DEV)
        gen.manual_seed(4)
        new = lambda n: torch.randn((n, 2, 128), generator=gen, device=DEV).to(torch.bfloat16)  # noqa: E731
        cache.extend(ints([0, 2]), ints([32, 30]))
        cache.append(new(62), new(62), ints([0, 2]), ints([0, 32, 62]))
        cache.fork(ints([0]), ints([1]))                       # pages: two shared, two of sequence 2, one left
        k, v, q = new(3), new(3), new(3).repeat_interleave(2, 1)

        def step():
            status = cache.extend()
            cache.append(k, v, status=status)
            return status, cache.attention(q)
        if captured:
            was = [t.clone() for t in (cache.pages, cache.page_table, cache.lengths, cache.refs)]
            step()
            for t, w in zip((cache.pages, cache.page_table, cache.lengths, cache.refs), was):
                t.copy_(w)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                status, got = step()
        lengths = [32, 32, 30]
        for i in range(6):
            k.copy_(new(3)), v.copy_(new(3))
            before = [held(cache, s) for s in range(3)]
            if captured:
                g.replay()
            else:
                status, got = step()
            # sequence 0 takes the last page; 1 and, once its second page is full, 2 are refused
            want = [0, 3, 0 if i < 2 else 3]
            assert status.tolist() == want
            lengths = [n + (s == 0) for n, s in zip(lengths, want)]
            assert cache.lengths.tolist() == lengths
            for s in range(3):
                for x, y in zip(held(cache, s), before[s]):
                    assert torch.equal(x[:, :y.shape[1]], y)   # what was there is still there
            ref, tol = kv_util.attention(cache, q, [0, 1, 2], [0, 1, 2, 3])
            assert bool(((got.double() - ref).abs() <= tol).all())


@pytest.mark.gpu
def test_rows_of_refused_items_stay_out_of_a_ragged_call():
    """Among served items, in any place, on both paths of the binding; a duplicate of an item is refused, so the first one's rows stay."""
    with Plan(96, 128, 1, 4, 0, 0.9) as plan:
        for path in (KVCache.append, binding._PYTHON_KV_METHODS["append"]):
            cache = KVCache.create(plan, 12, 3, 16, 5, 6, DEV)
            gen = torch.Generator(device=DEV)
            gen.manual_seed(8)
            seqs, counts = [3, 0, 3, 9, 1, 4], [20, 5, 7, 3, 97, 40]
            status = cache.extend(ints(seqs), ints(counts))
            assert status.tolist() == [0, 0, 5, 1, 4, 0]
            k, v = (torch.randn((sum(counts), 3, 96), generator=gen, device=DEV).to(torch.bfloat16) for _ in range(2))
            cu = [0, 20, 25, 32, 35, 132, 172]
            cache.pages.random_(0, 256, generator=gen)
            other = KVCache.create(plan, 12, 3, 16, 5, 6, DEV)
            for name in ("pages", "page_table", "lengths", "refs"):
                getattr(other, name).copy_(getattr(cache, name))
            path(cache, k, v, ints(seqs), ints(cu), status=status)
            rows = [t for i in (0, 1, 5) for t in range(cu[i], cu[i + 1])]
            other.append(k[rows].contiguous(), v[rows].contiguous(), ints([3, 0, 4]), ints([0, 20, 25, 65]))
            assert torch.equal(cache.pages, other.pages)
        with pytest.raises(ValueError):
            cache.append(k, v, ints(seqs), ints(cu), status=status[:5])
        with pytest.raises((TypeError, ValueError)):
            cache.append(k, v, ints(seqs), ints(cu), status=status.long())
