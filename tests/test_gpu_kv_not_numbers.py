"""Rows and scales of the paged KV cache that are no numbers: what sees them is NaN, and nothing else is."""
import pytest
import torch

import kv_util
from kv_util import DEV, filled
from paper_2504_13989_b200 import Plan
from paper_2504_13989_b200 import build as gbs_build

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def check_seen(cache, at, q, count, want, tol, **kw):
    """The rows of sequence 0 that see token `at` of KV head 1 are NaN, the others as they were."""
    group = q.shape[1] // 2
    got = cache.attention(q, ints(0), ints(0, count), count, **kw).double()
    pos = torch.arange(int(cache.lengths[0]) - count, int(cache.lengths[0]), device=DEV)
    sees = pos >= at
    if kw.get("window"):
        sees &= at > pos - kw["window"]
    bad = torch.zeros((count, q.shape[1]), dtype=torch.bool, device=DEV)
    bad[sees, group:] = True
    assert bool(torch.isnan(got[bad]).all())
    assert bool(((got - want).abs() <= tol)[~bad].all())
    return int(sees.sum())


@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("count", [1, 3, 60, 150])
@pytest.mark.parametrize("which", [0, 1])
def test_a_row_with_a_nan(count, which, asym):
    """In a unit that every row sees whole (at 20), in one whose tokens a window hides (24 < at), and among the last tokens."""
    gbs_build.build()
    with Plan(128, 128, 1, 4, 128, 0.9, asymmetric=asym) as plan:
        for at in (20, 70, 198):
            cache = filled(plan, [200], 2, 32, seed=at)
            gen = torch.Generator(device=DEV)
            gen.manual_seed(count)
            q = torch.randn((count, 4, 128), generator=gen, device=DEV).to(torch.bfloat16)
            few = 2 * count <= 16
            x = [torch.randn((200, 2, 128), generator=gen, device=DEV).to(torch.bfloat16) for _ in range(2)]
            cache.append(*x, ints(0), ints(0, 200))
            refs = [kv_util.attention(cache, q, [0], [0, count], few=few, window=w) for w in (0, 176)]
            clean = cache.read(ints(0), ints(0, 200), 200)
            x[which][at, 1, 5 + at % 100] = NAN
            cache.append(*x, ints(0), ints(0, 200))
            got = cache.read(ints(0), ints(0, 200), 200)
            assert bool(torch.isnan(got[which][at, 1]).all())
            got[which][at, 1] = clean[which][at, 1]
            assert torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1])
            assert check_seen(cache, at, q, count, *refs[0]) > 0
            seen = check_seen(cache, at, q, count, *refs[1], window=176)
            assert count > 1 or (seen == 0) == (at == 20)


@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("count", [1, 3, 60, 150])
def test_a_scale_that_is_no_number(count, asym):
    """In the pool itself: Delta (and lo) of a key or a value, in a unit that every row sees whole and in ones that they see in part."""
    gbs_build.build()
    with Plan(128, 128, 1, 4, 128, 0.9, asymmetric=asym) as plan:
        sf = 2 if asym else 1
        gen = torch.Generator(device=DEV)
        gen.manual_seed(count)
        cache = filled(plan, [200], 2, 32, seed=2)
        q = torch.randn((count, 4, 128), generator=gen, device=DEV).to(torch.bfloat16)
        refs = [kv_util.attention(cache, q, [0], [0, count], few=2 * count <= 16, window=w) for w in (0, 176)]
        for at in (20, 40, 199):
            block = cache.pages[cache.page_table[0, at // 32].long()].view(2, -1)[1]
            floats = block[32 * 128:].view(torch.float32)
            for which in range(2):
                for part in range(sf):
                    i = (which * 32 + at % 32) * sf + part
                    was = floats[i].clone()
                    for bad in (NAN, INF, -INF):
                        floats[i] = bad
                        assert check_seen(cache, at, q, count, *refs[0]) > 0
                        check_seen(cache, at, q, count, *refs[1], window=176)
                    floats[i] = was


@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("count", [1, 40])
def test_a_row_with_an_infinity(count, asym):
    """Appended: its scale is infinite or a NaN, and the rows that see it are NaN."""
    gbs_build.build()
    with Plan(128, 128, 1, 4, 128, 0.9, asymmetric=asym) as plan:
        gen = torch.Generator(device=DEV)
        gen.manual_seed(count)
        q = torch.randn((count, 4, 128), generator=gen, device=DEV).to(torch.bfloat16)
        for which in range(2):
            for at, where in ((20, (0,)), (70, (64,)), (199, (3, 77))):
                cache = filled(plan, [200], 2, 32, seed=at)
                x = [torch.randn((200, 2, 128), generator=gen, device=DEV).to(torch.bfloat16) for _ in range(2)]
                cache.append(*x, ints(0), ints(0, 200))
                ref = kv_util.attention(cache, q, [0], [0, count], few=2 * count <= 16)
                for sign in (INF, -INF):
                    for i in where:
                        x[which][at, 1, i] = sign
                    cache.append(*x, ints(0), ints(0, 200))
                    assert not torch.isfinite(cache.read(ints(0), ints(0, 200), 200)[which][at, 1]).any()
                    assert check_seen(cache, at, q, count, *ref) > 0
