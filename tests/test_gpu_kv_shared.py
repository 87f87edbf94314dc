"""gbs_kv_shared_attention against the plain implementation in 64 bits: groups of forks, groups that share nothing, and what lies between."""
import pytest
import torch

import kv_util
from kv_util import DEV, filled
from paper_2504_13989_b200 import GbsError, Plan
from paper_2504_13989_b200 import build as gbs_build

pytestmark = pytest.mark.gpu
LONG = 1 << 27                     # a prefix that is said to be so long is worth sharing, whatever it is


@pytest.fixture(scope="module", autouse=True)
def built():
    gbs_build.build()


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def rows(n, heads, d, seed, scale=1.0):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return (torch.randn((n, heads, d), generator=gen, device=DEV) * scale).to(torch.bfloat16)


def cu_of(counts):
    cu = [0]
    for c in counts:
        cu.append(cu[-1] + c)
    return cu


def forked(plan, prompts, forks, own, kvh, page, seed=0):
    """prompts: tokens of each prompt; forks: prompt of each further sequence; own: tokens that each of those gets behind it.  Sequences: the prompts,
    then the forks."""
    spare = sum(-(-(o + page) // page) for o in own) + 3
    cache = filled(plan, prompts + [0] * len(forks), kvh, page, seed, spare)
    wide = torch.full((cache.page_table.shape[0], cache.page_table.shape[1] + max(own, default=0) // page + 2), -1, dtype=torch.int32, device=DEV)
    wide[:, :cache.page_table.shape[1]] = cache.page_table
    from paper_2504_13989_b200 import KVCache
    cache = KVCache(plan, cache.pages, wide, cache.lengths, cache.refs, kvh, page)
    if forks:
        dst = ints(range(len(prompts), len(prompts) + len(forks)))
        assert cache.fork(ints(forks), dst).eq(0).all()
        assert cache.extend(dst, ints(own)).eq(0).all()
        n = sum(own)
        cache.append(rows(n, kvh, plan.info.d, seed + 1), rows(n, kvh, plan.info.d, seed + 2), dst, ints(cu_of(own)))
    return cache


def check(cache, q, seqs, cu, groups, causal=True, scale=0.0, **kw):
    got = cache.shared_attention(q, ints(seqs), ints(cu), None if groups is None else ints(groups), kw.pop("max_tokens", max(b - a for a, b in zip(cu, cu[1:]))),
                                 causal=causal, scale=scale, **{"max_prefix": LONG, **kw})
    want, tol = kv_util.attention(cache, q, seqs, cu, causal, 0, scale, few=False)
    live = ~want.isnan().all(-1).all(-1)
    assert bool(((got.double() - want).abs() <= tol)[live].all()), float(((got.double() - want).abs() / tol)[live].max())
    assert cache.plan.device_status() == 0
    return got


@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("d,kvh,group,page,prompt,count", [
    (128, 2, 4, 16, 300, 1),       # the rows of a prefix in tiles of 8 (up to 32 of them), and of a prompt
    (128, 1, 8, 64, 1000, 1),
    (80, 3, 1, 32, 517, 3),
    (128, 2, 4, 128, 900, 40),     # many rows of an item as well
    (96, 1, 7, 16, 95, 21),
    (8, 4, 2, 64, 64, 1),
    (128, 2, 3, 16, 17, 2),        # one page and a token
])
def test_forks_of_one_prompt(d, kvh, group, page, prompt, count, asym):
    n = 7
    own = [count + 13 * i for i in range(n)]
    with Plan(d, 128, 1, 4, 128, 0.9, asymmetric=asym) as plan:
        cache = forked(plan, [prompt], [0] * n, own, kvh, page)
        for items in (n, 2, 1):                                # 1: nothing is shared with anybody
            seqs = [1 + (3 * i) % n for i in range(items)]
            q = rows(items * count, kvh * group, d, 5, 3.0)
            check(cache, q, seqs, cu_of([count] * items), None)
            check(cache, q, seqs, cu_of([count] * items), [0, items], causal=False, scale=0.3, max_own=max(own) + page)
            for prefix in (0, prompt):                         # as the call judges itself: prefixes as short as these are not shared
                got = check(cache, q, seqs, cu_of([count] * items), None, max_prefix=prefix)
                # (many rows: with cached coordinates that are rounded once here)
                assert count * group > 16 or torch.equal(got, cache.attention(q, ints(seqs), ints(cu_of([count] * items)), count))


@pytest.mark.parametrize("count", [1, 30])
def test_groups_of_every_kind(count):
    """Forks of three prompts, one alone, unlike ones in a group, an item without tokens, one whose sequence there is not, one of no group."""
    prompts = [700, 40, 2000, 333]
    forks = [0, 0, 0, 1, 1, 2, 2, 2, 2]
    own = [31 + 7 * i for i in range(len(forks))]
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = forked(plan, prompts, forks, own, 2, 32, seed=3)
        seqs = [4, 5, 6, 3, 7, 8, 9, 99, 10, 11, 12, 4, 9, 0]
        counts = [count] * len(seqs)
        counts[5] = 0
        q = rows(sum(counts), 8, 128, 7, 2.0)
        for groups in ([0, 3, 4, 6, 11, 13], [0, 3, 3, 11], [2, 7, 11], [0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13, 14], None):
            out = torch.full_like(q, 7.0)
            got = cache.shared_attention(q, ints(seqs), ints(cu_of(counts)), None if groups is None else ints(groups), max(count, 1), max_prefix=LONG, out=out)
            keep = [i for i in range(len(seqs)) if seqs[i] < 13]
            want, tol = kv_util.attention(cache, q, [s if s < 13 else 0 for s in seqs], cu_of(counts), few=False)
            cu = cu_of(counts)
            for i in range(len(seqs)):
                a, b = cu[i], cu[i + 1]
                if i in keep:
                    assert bool(((got[a:b].double() - want[a:b]).abs() <= tol[a:b]).all()), (groups, i)
                else:
                    assert got[a:b].eq(0).all()                 # a sequence out of range: rows that see nothing


def test_pages_that_differ_in_the_middle_end_the_prefix():
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = filled(plan, [640, 640, 640], 1, 16, seed=9)
        cache.page_table[1, :20] = cache.page_table[0, :20]
        cache.page_table[1, 21:30] = cache.page_table[0, 21:30]
        cache.page_table[2, :39] = cache.page_table[0, :39]
        q = rows(3, 4, 128, 2, 2.0)
        check(cache, q, [0, 1, 2], [0, 1, 2, 3], None)
        check(cache, q, [2, 0, 1], [0, 1, 2, 3], [0, 2, 3])


def test_a_page_that_is_none_of_the_pools_is_left_out_of_a_prefix():
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = forked(plan, [256], [0, 0, 0, 0], [5, 6, 7, 8], 2, 16)
        q = rows(4, 8, 128, 2, 2.0)
        for bad in (-1, cache.pages.shape[0], 2 ** 31 - 1, -2 ** 31):
            cache.page_table[:, 3] = bad
            assert torch.allclose(cache.shared_attention(q, ints([1, 2, 3, 4]), max_prefix=LONG).float(), cache.attention(q, ints([1, 2, 3, 4])).float(), atol=0.02, rtol=0.02)


@pytest.mark.parametrize("which", [0, 1])
def test_scales_that_are_no_numbers_in_the_prefix(which):
    """A token of the prefix whose key (value) scale is a NaN: every row of the group is one, and no row of another group."""
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        for n in (3, 40):                                      # tiles of 8 rows and of 256
            cache = forked(plan, [300, 300], [0] * n + [1] * n, [9] * (2 * n), 1, 16)
            cache.pages.view(torch.float32).view(cache.pages.shape[0], -1)[int(cache.page_table[0, 4]), 16 * 32 + 16 * which + 5] = float("nan")
            q = rows(2 * n, 4, 128, 2)
            got = cache.shared_attention(q, ints(range(2, 2 + 2 * n)), None, ints([0, n, 2 * n]), max_prefix=LONG)
            assert got[:n].isnan().all() and got[n:].isfinite().all()
            assert plan.device_status() == 0


def test_broad_and_narrow_rows_where_the_two_parts_differ_much():
    """Scores that lie all in the prefix, or all behind it: the other part's share vanishes without a trace."""
    with Plan(128, 128, 1, 4, 128, 1.0) as plan:
        cache = forked(plan, [512], [0] * 12, [40] * 12, 1, 64)
        q = rows(12, 4, 128, 3)
        for scale in (0.0, 1e-6, 4.0, -4.0):
            check(cache, q, list(range(1, 13)), list(range(13)), None, scale=scale)


def test_strides_and_rows_that_are_left():
    with Plan(96, 128, 1, 4, 128, 0.9) as plan:
        cache = forked(plan, [200], [0] * 5, [30] * 5, 2, 16)
        counts = [4, 9, 1, 0, 3]
        cu = cu_of(counts)
        wide = rows(cu[-1] + 6, 8, 200, 4)
        q = wide[:, :, 8:104]
        room = torch.full((cu[-1] + 6, 11, 104), 5.0, dtype=torch.bfloat16, device=DEV)
        out = room[:, 2:10, :96]
        got = cache.shared_attention(q, ints([1, 2, 3, 4, 5]), ints(cu), None, 4, max_prefix=LONG, out=out)
        want, tol = kv_util.attention(cache, q[:cu[-1]].contiguous(), [1, 2, 3, 4, 5], cu, few=False)
        there = torch.zeros(cu[-1] + 6, dtype=torch.bool, device=DEV)
        for i, c in enumerate(counts):
            there[cu[i]:cu[i] + min(c, 4)] = True               # an item's tokens beyond max_tokens are left
        assert bool(((got[:cu[-1]].double() - want).abs() <= tol)[there[:cu[-1]]].all())
        assert got[~there].eq(5).all()
        room[:, 2:10, :96] = 5
        assert room.eq(5).all()                                # nothing beside the rows was written


def test_a_captured_step_that_grows():
    """A decoding step of forks, captured once: the sequences grow, and one is replaced by a fork of another prompt, without the host."""
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = forked(plan, [400, 90], [0] * 6, [3] * 6, 2, 16)
        seqs, side = ints(range(2, 8)), torch.cuda.Stream()
        k, v, q = rows(6, 2, 128, 1), rows(6, 2, 128, 2), rows(6, 8, 128, 3)

        def step():
            status = cache.extend(seqs)
            cache.append(k, v, seqs, status=status)
            return cache.shared_attention(q, seqs, max_own=32, max_prefix=LONG)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step()
        for i in range(8):
            if i == 4:
                cache.free(ints([4]))
                cache.fork(ints([1]), ints([4]))
                assert cache.lengths[4] == 90
            k.copy_(rows(6, 2, 128, 10 + i))
            q.copy_(rows(6, 8, 128, 20 + i))
            graph.replay()
            want, tol = kv_util.attention(cache, q, list(range(2, 8)), list(range(7)), few=False)
            assert bool(((out.double() - want).abs() <= tol).all())
        del graph


def test_two_calls_at_the_same_time():
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = forked(plan, [6000], [0] * 20, [200] * 20, 2, 64)
        side, seqs = torch.cuda.Stream(), ints(range(1, 21))
        qs = [rows(20, 16, 128, 5), rows(20, 16, 128, 6)]
        want = [cache.shared_attention(q, seqs, max_prefix=LONG) for q in qs]
        torch.cuda.synchronize()
        for _ in range(10):
            got = []
            for _ in range(3):
                got.append(cache.shared_attention(qs[0], seqs, max_prefix=LONG))
                got.append(cache.shared_attention(qs[1], seqs, max_prefix=LONG, stream=side))
            torch.cuda.synchronize()
            assert all(torch.equal(g, want[i & 1]) for i, g in enumerate(got))


def test_many_items_and_numbers_of_groups_that_fall():
    """8192 items in groups; then groups whose numbers are in no order, which may give any numbers but nothing beyond the rows."""
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = forked(plan, [100, 60], [0, 0, 1, 1], [5, 6, 7, 8], 1, 16)
        seqs = ([2, 3, 2, 3] * 2 + [4, 5] * 4) * 512
        q = rows(8192, 2, 128, 1)
        groups = sorted(list(range(0, 8192, 16)) + list(range(8, 8192, 16))) + [8192]
        got = cache.shared_attention(q, ints(seqs), None, ints(groups), max_prefix=LONG)
        assert torch.allclose(got.float(), cache.attention(q, ints(seqs)).float(), atol=0.02, rtol=0.02)
        room = torch.full((8200, 2, 128), 3.0, dtype=torch.bfloat16, device=DEV)
        for bad in ([5, 2, 9, 1, 30], [-7, 100, 50, 9000, 8192], [2 ** 31 - 1, -2 ** 31, 0, 8192]):
            cache.shared_attention(q, ints(seqs), None, ints(bad), max_prefix=LONG, out=room[:8192])
            assert room[8192:].eq(3).all() and plan.device_status() == 0


def test_the_native_call_and_the_one_in_python_agree_and_refuse():
    from paper_2504_13989_b200 import binding
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = forked(plan, [100], [0, 0], [5, 6], 1, 16)
        q = rows(2, 4, 128, 1)
        f = binding._PYTHON_KV_METHODS["shared_attention"]
        assert torch.equal(f(cache, q, ints([1, 2])), cache.shared_attention(q, ints([1, 2])))
        with pytest.raises(GbsError):
            cache.shared_attention(q, ints([1, 2]), out=q)
        with pytest.raises(TypeError):
            cache.shared_attention(q, ints([1, 2]), groups=torch.zeros(2, device=DEV))
        with pytest.raises(ValueError):
            cache.shared_attention(q, ints([1, 2]), groups=torch.zeros(2, dtype=torch.int32))
        with pytest.raises(TypeError):
            cache.shared_attention(q.float(), ints([1, 2]))
