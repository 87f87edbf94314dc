"""gbs_kv_evict over all ways in which a row (an item's KV head) is looked through: by 256 threads, by 1024, by clusters, and by one block of a cluster."""
import pytest
import torch

from kv_util import DEV, filled
from paper_2504_13989_b200 import KVCache, Plan
from paper_2504_13989_b200 import build as gbs_build
from test_gpu_kv_evict import check, ints, weights

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    gbs_build.build()


def wide(cache, tokens):
    """The same pool with a table that has room for sequences of so many tokens."""
    table = torch.full((cache.page_table.shape[0], -(-tokens // cache.page_size)), -1, dtype=torch.int32, device=DEV)
    table[:, :cache.page_table.shape[1]] = cache.page_table
    return KVCache(cache.plan, cache.pages, table, cache.lengths, cache.refs, cache.n_kv_heads, cache.page_size)


def best(mass, lengths, keep, recent, first):
    """[items, heads, keep] positions, by a stable sort; weights without NaN."""
    out = []
    for i, n in enumerate(lengths):
        w = mass[i, :, first:n - recent] + 0.0
        p = w.argsort(dim=-1, descending=True, stable=True)[:, :keep - first - recent].sort(-1).values + first
        ends = [torch.arange(a, b, device=DEV).expand(w.shape[0], -1) for a, b in ((0, first), (n - recent, n))]
        out.append(torch.cat([ends[0], p, ends[1]], -1))
    return torch.stack(out)


@pytest.mark.parametrize("seqs,heads,lengths,room", [
    (20, 8, [30000], 0),                                       # more rows than SMs, and long
    (2, 8, [20000, 16385], 0),
    (38, 8, [9001, 4097], 0),
    (6, 8, [300], 130000),                                     # short ones where there is room for long ones
    (5, 8, [40000, 300, 16384, 16385, 150], 130000),           # both in one call
    (1, 3, [130001], 0),
    (100, 8, [301, 4096], 60000),
])
def test_rows(seqs, heads, lengths, room):
    keep, recent, first = 100, 30, 4
    lengths = [lengths[i % len(lengths)] for i in range(seqs)]
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = filled(plan, lengths, heads, 64, seed=1, spare=2 * seqs)
        if room:
            cache = wide(cache, room)
        for kind in ("few", "plain"):
            mass = weights(cache, max(lengths), 3, kind)
            was, into = [t.clone() for t in (cache.page_table, cache.lengths, cache.refs)], torch.zeros_like(mass)
            status, kept = cache.evict(mass, keep, recent=recent, first=first, into=into)
            assert status.eq(0).all() and cache.lengths.eq(keep).all()
            want = best(mass, lengths, keep, recent, first)
            assert torch.equal(kept.long(), want)
            assert torch.equal(into[..., :keep], mass.gather(-1, want)) and into[..., keep:].eq(0).all()
            assert int(cache.refs.sum()) == 2 * seqs
            for t, w in zip((cache.page_table, cache.lengths, cache.refs), was):
                t.copy_(w)


def test_one_block_of_a_cluster_against_the_model():
    """Bytes, tables and refused items as well, with weights of every kind, where single blocks and clusters work side by side."""
    with Plan(128, 128, 1, 4, 128, 0.9, asymmetric=True) as plan:
        for kind in ("few", "any", "same"):
            cache = wide(filled(plan, [17000, 600, 40, 16384], 1, 128, seed=2, spare=8), 200000)
            w = weights(cache, 17000, 5, kind)
            check(cache, w, 200, [1, 0, 9, 3, 0, 2], 20, 3, into=weights(cache, 17000, 6), statuses=[0, 0, 1, 0, 5, 0])


@pytest.mark.parametrize("items", [255, 256, 257])
def test_pages_looked_for_beside_and_before(items):
    """Around the number of items from which the search for pages is a launch of its own; pages run out before the end, and the last item names a sequence again."""
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = filled(plan, [17 + i % 30 for i in range(items)], 2, 16, seed=1, spare=200)
        seqs = list(range(items))[::-1]
        seqs[-1] = seqs[0]
        w = weights(cache, 50, 3, "few")
        status = check(cache, w, 20, seqs, 3, 2, into=weights(cache, 50, 4))
        assert status.eq(3).any() and int(status[-1]) == 5
