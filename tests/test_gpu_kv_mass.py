"""gbs_kv_attention_mass against the formula in 64 bits."""
import pytest
import torch

import kv_util
from kv_util import DEV, filled
from paper_2504_13989_b200 import GbsError, Plan
from paper_2504_13989_b200 import build as gbs_build

pytestmark = pytest.mark.gpu


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


def wanted(cache, q, seqs, cu, base, decay, mass, causal=True, window=0, scale=0.0, most=1 << 30):
    """(result, tolerance) in 64 bits.

    A row's score over token j is off by at most e = |scale| |q|_2 (|khat_j|_2 + sqrt(128) |mid_j|) 128 2^-24: seven stages of additions and the rounding to 24 bits of the largest
    coordinate put the rotated row off by 8 2^-24 |q|_2 in each of 128 coordinates (8 sqrt(128) = 91 of it as a vector); the integer's way to a float, the scale
    and the factors add 7 roundings of the product, and the middle of an asymmetric row, a sum of its own, as many.  Where z - m is formed it is rounded, by 2^-24 of
    |z - m| <= 150 at most, below which nothing is left; log2 to e: 2^-24 150 / 1.44.  A probability is a quotient of which both sides are off by that, by ex2 (2^-22)
    and by the additions of a row's sum, of which a thread makes one for each 128 tokens, two for each unit, ten at the end; the sum over rows is compensated
    (2^-22), and the old mass times decay is rounded once.  What underflows adds 1e-36."""
    d, kvh = cache.plan.info.d, cache.n_kv_heads
    heads = q.shape[1]
    group = heads // kvh
    want, tol = mass.double().clone(), torch.zeros(mass.shape, dtype=torch.float64, device=DEV)
    scale = scale or d ** -0.5
    for i, seq in enumerate(seqs):
        count = cu[i + 1] - cu[i]
        if count == 0 or not 0 <= seq < len(cache.lengths) or int(cache.lengths[seq]) == 0:
            continue
        length = int(cache.lengths[seq])
        x = torch.zeros((count, heads, 128), dtype=torch.float64, device=DEV)
        x[..., :d] = q[cu[i]:cu[i + 1]].double()
        x = (x @ kv_util.h128() / 128 ** 0.5).view(count, kvh, group, 128)[:most]
        k, _, km, _ = kv_util.rows_of(cache, seq, middles=True)
        width = min(mass.shape[2], length)
        new, lim = torch.zeros(kvh, length, dtype=torch.float64, device=DEV), torch.zeros(kvh, length, dtype=torch.float64, device=DEV)
        for a in range(0, x.shape[0], 64):
            y = x[a:a + 64]
            s = torch.einsum("qhgd,hkd->qhgk", y, k) * scale
            pos = (length - count + a + torch.arange(y.shape[0], device=DEV))[:, None]
            t = torch.arange(length, device=DEV)
            seen = (t <= pos) if causal else (t < length) & (pos > -length - count)
            if window:
                seen = seen & (t > pos - window)
            seen = seen[:, None, None]
            s = s.masked_fill(~seen, float("-inf"))
            top = s.amax(-1, keepdim=True)
            p = torch.where(seen, torch.exp(s - torch.where(top == float("-inf"), torch.zeros_like(top), top)), 0.0)
            total = p.sum(-1, keepdim=True)
            p = torch.where(total == 0, torch.zeros_like(p), p / total)
            e = abs(scale) * y.norm(dim=-1)[..., None] * (k.norm(dim=-1) + 128 ** 0.5 * km)[None, :, None] * 128 * 2.0 ** -24
            e = torch.where(seen, e, 0.0)
            # the denominator is off by the mean of the e of its tokens at most by the largest of them
            rel = e + e.amax(-1, keepdim=True) + 2 * 2.0 ** -24 * 105 + 2.0 ** -20 + (3 * length / 128 + 12) * 2.0 ** -24
            new += p.sum((0, 2))
            lim += (p * rel).sum((0, 2))
        old = torch.zeros_like(new)
        if decay:
            n = max(0, min(length - count, width))
            old[:, :n] = base[seq, :, :n].double() * decay
        want[seq, :, :width] = (old + new)[:, :width]
        tol[seq, :, :width] = (lim + 2.0 ** -22 * (old + new).abs() + 1e-36)[:, :width]
    return want, tol


def check(cache, q, seqs, cu, width=None, decay=1.0, own_base=True, most=None, **kw):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(11)
    width = width or int(cache.lengths.max()) + 5
    mass = torch.rand((len(cache.lengths), cache.n_kv_heads, width), generator=gen, device=DEV)
    base = mass if own_base else torch.rand(mass.shape, generator=gen, device=DEV)
    want, tol = wanted(cache, q, seqs, cu, base.clone(), decay, mass, most=most or 1 << 30, **kw)
    got = cache.attention_mass(q, mass, ints(seqs), ints(cu), most or max(max(b - a for a, b in zip(cu, cu[1:])), 1), decay=decay,
                               base=None if own_base else base, **kw)
    assert got is mass
    off = (got.double() - want).abs()
    assert bool((off <= tol).all()), float((off / tol.clamp(min=1e-300)).max())
    assert cache.plan.device_status() == 0
    return got


@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("d,kvh,group,page,lengths,counts", [
    (128, 2, 4, 64, [300], [1]),
    (128, 8, 1, 16, [1, 2, 17, 129, 640, 4000], [1, 1, 1, 1, 1, 1]),
    (80, 3, 7, 32, [517, 33, 128], [3, 2, 1]),
    (128, 1, 16, 128, [900, 1000, 1], [1, 1, 1]),             # a whole pass of sixteen rows, and a second one
    (128, 1, 17, 128, [900, 127], [1, 1]),
    (96, 2, 4, 16, [700, 256], [40, 256]),                    # chunks, and a prompt from its first token
    (8, 1, 2, 64, [5000, 65], [130, 65]),
    (128, 2, 2, 16, [16, 48, 0, 30], [16, 0, 1, 30]),         # an item without tokens, and one without a sequence to speak of
])
def test_weights(d, kvh, group, page, lengths, counts, asym):
    with Plan(d, 128, 1, 4, 128, 0.9, asymmetric=asym) as plan:
        cache = filled(plan, lengths, kvh, page, seed=d)
        order = list(range(len(lengths)))[::-1]
        cu = cu_of([counts[s] for s in order])
        q = rows(cu[-1], kvh * group, d, 3, 3.0)
        check(cache, q, order, cu)
        check(cache, q, order, cu, decay=0.9, own_base=False, causal=False, scale=-0.2)
        check(cache, q, order, cu, decay=0.0, window=20)
        check(cache, q, order, cu, width=31, decay=0.5, window=200, scale=1.5)


def test_long_sequences_and_many_rows():
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = filled(plan, [60000, 3000, 20000], 2, 64, seed=2)
        check(cache, rows(3, 8, 128, 1, 2.0), [0, 1, 2], [0, 1, 2, 3])
        check(cache, rows(640, 4, 128, 1, 2.0), [2, 1], [0, 40, 640], decay=0.99)
        check(cache, rows(64, 4, 128, 2, 2.0), [0], [0, 64], decay=0.0, window=5000)


@pytest.mark.parametrize("count,n", [(1, 3000), (9, 1100)])
def test_many_items(count, n):
    """More items than the threads that look through them; few query rows, and many."""
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = filled(plan, [9 + i % 140 for i in range(n)], 1, 16, seed=2)
        counts = [count if i % 17 else 0 for i in range(n)]
        check(cache, rows(sum(counts), 4, 128, 1, 2.0), list(range(n))[::-1], cu_of(counts), decay=0.5)


@pytest.mark.parametrize("count,heads", [(1, 4), (7, 16), (30, 8), (90, 8)])
def test_windows_of_queries_that_see_all_that_follows(count, heads):
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = filled(plan, [2000, 129, 90], 2, 64, seed=2)
        for window in (1, 50, 129, 1 << 30):
            check(cache, rows(3 * count, heads, 128, 1, 2.0), [0, 1, 2], cu_of([count] * 3), causal=False, window=window)
            check(cache, rows(3 * count, heads, 128, 1, 2.0), [0, 1, 2], cu_of([count] * 3), window=window, decay=0.0)


def test_scores_that_have_no_room():
    """A width by which the scores of a call are not kept: the second pass finds them again."""
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = filled(plan, [700, 3000, 1, 64], 2, 64, seed=2)
        for count, heads in ((1, 64), (4, 16), (1, 2)):
            width = (256 << 20) // (4 * 2 * 4 * (count * heads // 2 + (count * heads // 2) % 2)) + 1
            counts = [count, count, 1, count]
            check(cache, rows(sum(counts), heads, 128, 1, 2.0), [0, 1, 2, 3], cu_of(counts), width=width, decay=0.9, window=2000)


def test_tokens_beyond_max_tokens_give_no_weight():
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = filled(plan, [200, 90], 2, 16, seed=2)
        q = rows(29, 4, 128, 1, 2.0)
        check(cache, q, [0, 1], [0, 20, 29], most=12)
        check(cache, q, [0, 1], [0, 20, 29], most=1)


def test_strides_rows_behind_and_sequences_out_of_range():
    with Plan(96, 128, 1, 4, 128, 0.9) as plan:
        cache = filled(plan, [200, 90, 300], 2, 16, seed=2)
        wide = rows(9, 6, 200, 4)
        q = wide[:, 1:5, 8:104]
        check(cache, q, [2, 99, 0, -1], [0, 3, 5, 6, 7])
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = filled(plan, [200, 90], 2, 16, seed=2)
        mass = torch.full((2, 2, 300), 4.0, device=DEV)
        cache.attention_mass(rows(2, 4, 128, 1), mass, ints([1, 7]), decay=0.0)
        assert mass[0].eq(4).all() and mass[1, :, 90:].eq(4).all() and abs(float(mass[1, 0, :90].sum()) - 2) < 1e-4


def test_the_weights_of_a_row_add_up():
    """Sixteen query heads on one KV head: the weights of a token's queries add up to 16, whatever the scale; NaN and infinity in the old weights stay where they are."""
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = filled(plan, [3000], 1, 32, seed=2)
        for scale in (0.0, 1e-30, 100.0, -100.0):
            mass = torch.zeros((1, 1, 3000), device=DEV)
            mass[0, 0, 5], mass[0, 0, 6], mass[0, 0, 2999] = float("nan"), float("inf"), float("nan")
            cache.attention_mass(rows(1, 16, 128, 1), mass, scale=scale)
            assert mass[0, 0, 5].isnan() and mass[0, 0, 6].isinf()
            mass[0, 0, 5] = mass[0, 0, 6] = 0
            assert mass.isfinite().all()
            clean = cache.attention_mass(rows(1, 16, 128, 1), torch.full((1, 1, 3000), float("nan"), device=DEV), scale=scale, decay=0.0)
            # 3000 weights, each off by at most what the tolerance above has for scores of a hundred (2^-13), their sum in 64 bits
            assert abs(float(clean.double().sum()) - 16) < 16 * 2.0 ** -13


@pytest.mark.parametrize("count", [1, 20])
def test_scales_that_are_no_numbers(count):
    """A key scale that is a NaN or infinite makes what the rows see NaN; value scales, tokens that no row sees and other sequences count for nothing."""
    for bad in (float("nan"), float("inf"), -float("inf")):
        with Plan(128, 128, 1, 4, 128, 0.9) as plan:
            cache = filled(plan, [300, 300], 1, 16, seed=2)
            f = cache.pages.view(torch.float32).view(cache.pages.shape[0], -1)
            f[int(cache.page_table[0, 4]), 16 * 32 + 16 + 5] = bad                     # a value's
            q = rows(2 * count, 4, 128, 2)
            cu = ints([0, count, 2 * count])
            mass = cache.attention_mass(q, torch.zeros((2, 1, 300), device=DEV), None, cu, count)
            assert mass.isfinite().all()
            f[int(cache.page_table[0, 4]), 16 * 32 + 5] = bad                          # token 69's key
            mass = cache.attention_mass(q, torch.zeros((2, 1, 300), device=DEV), None, cu, count)
            assert mass[0].isnan().all() and mass[1].isfinite().all()
            mass = cache.attention_mass(q, torch.zeros((2, 1, 300), device=DEV), None, cu, count, window=100)
            assert mass.isfinite().all() and mass[0, 0, :181].eq(0).all()


@pytest.mark.parametrize("count", [1, 5, 40])
@pytest.mark.parametrize("asym", [False, True])
def test_pages_without_a_number_among_their_scales(count, asym):
    """Whole pages of NaN, the first that a thread sees among them, make what the rows see NaN as well."""
    with Plan(128, 128, 1, 4, 128, 0.9, asymmetric=asym) as plan:
        for pages in ((0,), (4,), (0, 1, 2, 3), (8, 9, 10, 11), (18,)):
            cache = filled(plan, [300, 300], 1, 16, seed=2)
            f = cache.pages.view(torch.float32).view(cache.pages.shape[0], -1)
            for p in pages:
                f[int(cache.page_table[0, p]), 16 * 32:16 * 32 + (32 if asym else 16)] = float("nan")
            q = rows(2 * count, 4, 128, 2)
            mass = cache.attention_mass(q, torch.zeros((2, 1, 300), device=DEV), None, ints([0, count, 2 * count]), count, causal=False)
            assert mass[0].isnan().all() and mass[1].isfinite().all()


def test_a_page_that_is_none_of_the_pools():
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = filled(plan, [300], 2, 16, seed=2)
        cache.page_table[0, 3] = 2 ** 30
        mass = cache.attention_mass(rows(1, 8, 128, 2), torch.ones((1, 2, 300), device=DEV))
        assert mass[:, :, 48:64].eq(1).all() and abs(float(mass.double().sum()) - 2 * 299 - 8) < 1e-3


def test_a_captured_step_and_two_calls_at_the_same_time():
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = filled(plan, [5000, 300, 40], 2, 64, seed=2, spare=20)
        q, side = rows(3, 8, 128, 2), torch.cuda.Stream()
        mass = torch.zeros((3, 2, 6000), device=DEV)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            cache.attention_mass(q, mass)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cache.attention_mass(q, mass, decay=0.5)
        for i in range(3):
            q.copy_(rows(3, 8, 128, 30 + i))
            want, tol = wanted(cache, q, [0, 1, 2], [0, 1, 2, 3], mass.clone(), 0.5, mass)
            graph.replay()
            assert bool(((mass.double() - want).abs() <= tol).all())
            cache.lengths -= 3                                  # the next step sees other lengths
        del graph
        qs = [rows(3, 8, 128, 5), rows(3, 8, 128, 6)]
        base = torch.rand((3, 2, 6000), device=DEV)
        want = [cache.attention_mass(q, torch.zeros_like(base), base=base) for q in qs]
        into = [[torch.zeros_like(base) for _ in range(3)] for _ in range(2)]
        torch.cuda.synchronize()
        for j in range(3):
            cache.attention_mass(qs[0], into[0][j], base=base)
            cache.attention_mass(qs[1], into[1][j], base=base, stream=side)
        torch.cuda.synchronize()
        assert all(torch.equal(t, want[i]) for i in range(2) for t in into[i])


def test_refusals():
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = filled(plan, [30, 30], 2, 16, seed=2)
        q, mass = rows(2, 4, 128, 1), torch.zeros((2, 2, 40), device=DEV)
        for bad in (mass[:, :, ::2], mass[:1], mass.double(), mass.cpu(), mass[:, :1]):
            with pytest.raises((ValueError, TypeError)):
                cache.attention_mass(q, bad)
            with pytest.raises((ValueError, TypeError)):
                cache.attention_mass(q, mass, base=bad)
        for kw in (dict(decay=float("nan")), dict(scale=float("inf")), dict(max_tokens=2), dict(window=-1)):
            with pytest.raises((GbsError, ValueError)):
                cache.attention_mass(q, mass, **kw)
        assert mass.eq(0).all()
