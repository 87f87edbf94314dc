"""gbs_kv_evict against a plain implementation on lists, byte for byte."""
import numpy as np
import pytest
import torch

import kv_util
from kv_util import DEV, Model, filled
from paper_2504_13989_b200 import GbsError, KVCache, Plan
from paper_2504_13989_b200 import build as gbs_build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    gbs_build.build()


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def rows(n, heads, d, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return torch.randn((n, heads, d), generator=gen, device=DEV).to(torch.bfloat16)


def tokens_of(cache, pages, seq_len):
    """[heads, tokens, bytes of a token] of a list of pages, from the pool's bytes `pages` on the host."""
    ps, sf = cache.page_size, 2 if cache.plan.info.asymmetric else 1
    b = cache.pages.cpu().numpy().reshape(cache.pages.shape[0], cache.n_kv_heads, -1)[pages]
    parts, at = [], 0
    for size in (64, 64, 4 * sf, 4 * sf):
        parts.append(b[:, :, at:at + ps * size].reshape(len(pages), cache.n_kv_heads, ps, size))
        at += ps * size
    return np.concatenate(parts, -1).transpose(1, 0, 2, 3).reshape(cache.n_kv_heads, len(pages) * ps, -1)[:, :seq_len]


def stay(w, length, keep, recent, first):
    """Positions that stay of one KV head's weights w (as long as the sequence): the largest, of two alike the lower position; NaN the largest of all."""
    key = np.where(np.isnan(w), np.inf, w.astype(np.float64))
    nan = np.isnan(w)
    between = sorted(range(first, length - recent), key=lambda p: (not nan[p], -key[p], p))[:keep - first - recent]
    return sorted(list(range(first)) + between + list(range(length - recent, length)))


def model_of(cache, spare_free=True):
    m = Model(cache.pages.shape[0], cache.page_size, len(cache.lengths), cache.page_table.shape[1])
    m.refs, m.lengths = cache.refs.tolist(), cache.lengths.tolist()
    table = cache.page_table.tolist()
    m.pages = [t[:-(-n // m.ps)] for t, n in zip(table, m.lengths)]
    return m


def check(cache, mass, keep, seqs, recent=0, first=0, into=None, statuses=None):
    m = model_of(cache)
    before = [tokens_of(cache, m.pages[s], m.lengths[s]) if m.lengths[s] else None for s in range(m.n_seqs)]
    w = mass.cpu().numpy()
    was = (mass if into is None else into).clone()
    shared = {p for s in range(m.n_seqs) for p in m.pages[s]}
    pool = cache.pages.clone()
    # the plain bookkeeping: pages for all that are cut, in order, then the old ones are let go
    need, seen, wishes = -(-keep // m.ps), set(), []
    for s in seqs:
        if not 0 <= s < m.n_seqs:
            wishes.append((1, 0))
        elif s in seen:
            wishes.append((5, 0))
        else:
            seen.add(s)
            wishes.append((0, need if m.lengths[s] > keep else 0))
    got = m._serve(wishes)
    want_status = [st if st else (0 if g is not None else 3) for (st, _), g in zip(wishes, got)]
    if statuses is not None:
        assert want_status == statuses
    status, kept = cache.evict(mass, keep, ints(seqs), recent=recent, first=first, into=into)
    assert status.tolist() == want_status
    kept, out = kept.cpu().numpy(), (mass if into is None else into).cpu().numpy()
    assert kept.shape == (len(seqs), cache.n_kv_heads, keep)
    was = was.cpu().numpy()
    for i, s in enumerate(seqs):
        if want_status[i]:
            assert (kept[i] == -1).all()
            continue
        n = m.lengths[s]
        wide = np.zeros((cache.n_kv_heads, max(n, w.shape[2])), np.float32)
        wide[:, :w.shape[2]] = w[s]
        for h in range(cache.n_kv_heads):
            p = list(range(n)) if n <= keep else stay(wide[h, :n], n, keep, recent, first)
            assert kept[i, h].tolist() == p + [-1] * (keep - len(p)), (i, h)
            k = min(len(p), w.shape[2])
            was[s, h, :k] = wide[h, p][:k]
        if n > keep:
            for p in m.pages[s]:
                m.refs[p] -= 1
            m.pages[s], m.lengths[s] = got[i], keep
    np.testing.assert_array_equal(out, was)
    m.check(cache)
    for i, s in enumerate(seqs):
        if want_status[i] == 0 and m.lengths[s]:
            now = tokens_of(cache, m.pages[s], m.lengths[s])
            for h in range(cache.n_kv_heads):
                p = kept[i, h][kept[i, h] >= 0]
                np.testing.assert_array_equal(now[h], before[s][h][p])
    for p in sorted(shared):                                   # what was held is as it was, whoever holds it now
        assert torch.equal(cache.pages[p], pool[p])
    return status


def weights(cache, width, seed, kind="few"):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    w = torch.rand((len(cache.lengths), cache.n_kv_heads, width), generator=gen, device=DEV)
    if kind == "few":                                          # many alike
        w = (w * 5).floor()
    elif kind == "any":
        w = torch.randint(-2 ** 31, 2 ** 31 - 1, w.shape, generator=gen, device=DEV, dtype=torch.int32).view(torch.float32)
    elif kind == "same":
        w = torch.zeros_like(w)
        w[..., ::3] = -0.0
    return w


@pytest.mark.parametrize("kind", ["few", "any", "same", "plain"])
@pytest.mark.parametrize("page,heads,asym,lengths,keep,recent,first", [
    (16, 2, False, [300, 16, 1, 0, 33, 32], 32, 8, 4),
    (32, 1, True, [1000, 31, 33, 999], 31, 0, 0),
    (64, 3, False, [700, 64, 65, 129], 65, 65, 0),             # nothing but the last ones
    (128, 2, True, [5000, 300], 257, 100, 157),                # nothing between
    (16, 1, False, [2, 3, 20000, 1], 1, 0, 0),
    (16, 8, False, [40, 30, 9000], 8191, 17, 3),
])
def test_what_stays(page, heads, asym, lengths, keep, recent, first, kind):
    with Plan(128, 128, 1, 4, 128, 0.9, asymmetric=asym) as plan:
        cache = filled(plan, lengths, heads, page, seed=keep, spare=len(lengths) * (-(-keep // page) + 1))
        order = list(range(len(lengths)))[::-1]
        w = weights(cache, max(lengths), keep, kind)
        into = torch.full_like(w, -3.0)
        check(cache, w, keep, order, recent, first, into=into)
        check(cache, w, keep, order, recent, first)            # all short enough by now
        cache = filled(plan, lengths, heads, page, seed=keep, spare=len(lengths) * (-(-keep // page) + 1))
        check(cache, w, keep, order, recent, first)            # in place


def test_weights_that_are_no_numbers():
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = filled(plan, [500, 400], 2, 16, seed=1, spare=20)
        w = weights(cache, 500, 1, "plain")
        w[0, 0, 100:130], w[0, 1, 50:60], w[1, 0, 7], w[1, 1] = float("nan"), float("inf"), -float("nan"), -float("inf")
        check(cache, w, 40, [0, 1], 3, 2)


def test_a_width_short_of_the_sequences():
    """Positions from the width on weigh 0, and have no place in the new weights either."""
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        for width in (1, 20, 100):
            cache = filled(plan, [500, 90], 2, 16, seed=1, spare=20)
            check(cache, weights(cache, width, 1, "plain") - 0.5, 40, [0, 1], 3, 2)


def test_long_sequences():
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = filled(plan, [131000, 70001], 1, 128, seed=1, spare=600)
        for kind in ("plain", "same"):
            check(cache, weights(cache, 131000, 2, kind), 20000 if kind == "plain" else 9999, [1, 0], 100, 4)


def test_long_sequences_of_which_the_ends_stay():
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        for recent, first in ((9000, 999), (9999, 0), (0, 9999)):
            cache = filled(plan, [131000, 70001, 9999], 2, 128, seed=1, spare=200)
            check(cache, weights(cache, 131000, 2, "plain"), 9999, [1, 2, 0], recent, first)


def test_forks_keep_what_they_share():
    """Two forks of a prompt are cut down, one after the other and in one call, and the prompt is what it was."""
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = filled(plan, [530, 0, 0], 2, 16, seed=1, spare=14)
        cache.fork(ints([0, 0]), ints([1, 2]))
        w = weights(cache, 600, 3, "plain")
        check(cache, w, 64, [2], 10, 4)
        check(cache, w, 64, [1], 10, 4)
        assert cache.refs.sum() == 34 + 4 + 4


def test_a_document_and_its_forks_in_one_call():
    """All read pages that the others let go."""
    with Plan(128, 128, 1, 4, 128, 0.9, asymmetric=True) as plan:
        cache = filled(plan, [530, 0, 0, 0], 2, 16, seed=1, spare=30)
        cache.fork(ints([0, 0, 0]), ints([1, 2, 3]))
        check(cache, weights(cache, 600, 3, "plain"), 64, [2, 0, 3, 1], 10, 4)
        assert cache.refs.sum() == 16


def test_a_page_that_is_none_of_the_pools():
    """What would stay of it becomes rows of zeros."""
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        for bad in (2 ** 31 - 1, -1, -2 ** 31):
            cache = filled(plan, [100], 2, 16, seed=1, spare=4)
            refs, page = cache.refs.clone(), int(cache.page_table[0, 2])
            cache.page_table[0, 2] = bad
            w = torch.zeros((1, 2, 100), device=DEV)
            w[0, :, 30:50] = 1.0
            status, kept = cache.evict(w, 20)
            assert status.item() == 0 and kept[0].tolist() == [list(range(30, 50))] * 2
            for x in cache.read(ints([0]), ints([0, 20]), 20):
                assert x[2:18].eq(0).all() and x[:2].ne(0).any() and x[18:].ne(0).any()
            refs -= refs.clamp(max=1)
            refs[page] = 1                                     # nobody let it go
            now = cache.refs.clone()
            now[cache.page_table[0, :2].long()] -= 1
            assert torch.equal(now, refs)


def test_items_that_are_refused():
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = filled(plan, [300, 200, 100, 20], 1, 16, seed=1, spare=3)
        w = weights(cache, 300, 3, "plain")
        # three pages are free: the first item that needs more than is left is refused, and so are those behind it that need any
        check(cache, w, 30, [0, 9, 1, 0, 3, 2, -1], 3, 2, statuses=[0, 1, 3, 5, 0, 3, 1])
        check(cache, w, 30, [1, 2], 3, 2, statuses=[0, 0])     # there is room now
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = filled(plan, [300, 200], 1, 16, seed=1, spare=1)
        check(cache, weights(cache, 300, 3, "plain"), 30, [0, 1], 3, 2, statuses=[3, 3])


def test_many_items():
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        n = 3000
        cache = filled(plan, [17 + i % 40 for i in range(n)], 1, 16, seed=1, spare=n)
        check(cache, weights(cache, 60, 3, "few"), 16, list(range(n))[::-1] + [5, 6] + [n], 2, 1)


def test_a_captured_step():
    """The sequences grow step by step and are cut down when they are longer than the budget, without the host."""
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = KVCache.create(plan, 40, 2, 16, 3, 12, DEV)
        k, v, q, mass = rows(3, 2, 128, 1), rows(3, 2, 128, 2), rows(3, 8, 128, 3), torch.zeros((3, 2, 100), device=DEV)

        def step():
            status = cache.extend()
            cache.append(k, v, status=status)
            out = cache.attention(q)
            cache.attention_mass(q, mass)
            return out, cache.evict(mass, 24, recent=4)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out, (status, kept) = step()
        twin = KVCache.create(plan, 40, 2, 16, 3, 12, DEV)
        for t, u in ((twin.pages, cache.pages), (twin.page_table, cache.page_table), (twin.lengths, cache.lengths), (twin.refs, cache.refs)):
            t.copy_(u)
        weight = mass.clone()
        for i in range(60):
            k.copy_(rows(3, 2, 128, 10 + i))
            q.copy_(rows(3, 8, 128, 20 + i))
            graph.replay()
            assert twin.extend().eq(0).all()
            twin.append(k, v)
            assert torch.equal(twin.attention(q), out)
            twin.attention_mass(q, weight)
            s, p = twin.evict(weight, 24, recent=4)
            assert torch.equal(s, status) and torch.equal(p, kept) and torch.equal(weight, mass)
            assert torch.equal(twin.page_table, cache.page_table) and torch.equal(twin.refs, cache.refs)
            assert cache.lengths.tolist() == [min(i + 2, 24)] * 3
        assert torch.equal(kv_util.rows_of(cache, 1)[0], kv_util.rows_of(twin, 1)[0])
        del graph


def test_attention_over_what_is_left():
    """After eviction attention is attention over the tokens that stay, KV head by KV head."""
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = filled(plan, [400], 2, 16, seed=1, spare=10)
        k, v = kv_util.rows_of(cache, 0)
        w = weights(cache, 400, 3, "plain")
        _, kept = cache.evict(w, 100, recent=10, first=2)
        q = rows(1, 8, 128, 5)
        want, tol = kv_util.attention(cache, q, [0], [0, 1])
        p = kept[0].long()
        for h in range(2):
            a, b = kv_util.rows_of(cache, 0)
            assert torch.equal(a[h], k[h, p[h]]) and torch.equal(b[h], v[h, p[h]])
        assert bool(((cache.attention(q).double() - want).abs() <= tol).all())


def test_refusals():
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = filled(plan, [30, 30], 2, 16, seed=2)
        mass = torch.zeros((2, 2, 40), device=DEV)
        for bad in (mass[:, :, ::2], mass[:1], mass.double(), mass.cpu(), mass[:, :1]):
            with pytest.raises((ValueError, TypeError)):
                cache.evict(bad, 5)
            with pytest.raises((ValueError, TypeError)):
                cache.evict(mass, 5, into=bad)
        for kw in (dict(keep=0), dict(keep=-3), dict(keep=5, recent=6), dict(keep=5, first=-1), dict(keep=5, recent=3, first=3)):
            with pytest.raises((GbsError, ValueError)):
                cache.evict(mass, **kw)
        assert cache.lengths.tolist() == [30, 30]
        status, kept = cache.evict(mass, 5, ints([]))
        assert status.numel() == 0 and kept.shape == (0, 2, 5)
