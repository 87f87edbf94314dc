"""Long contexts from end to end: a document that many answers start from, whose weights are kept, shared and cut down as the answers grow."""
import pytest
import torch

import kv_util
from kv_util import DEV
from paper_2504_13989_b200 import KVCache, Plan
from paper_2504_13989_b200 import build as gbs_build
from test_gpu_kv_evict import stay
from test_gpu_kv_mass import wanted

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def test_offsets_beyond_32_bits():
    """A pool of more than 4 GB whose last pages are the ones in use, and weights of more than 2^31 places: results as in a small pool."""
    gbs_build.build()
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        small = kv_util.filled(plan, [0, 0, 0, 700, 3000], 2, 64, 3, spare=20)
        here, total, narrow, wide = small.pages.shape[0], 260000, 3100, (1 << 28) + 7
        off = total - here
        pages = torch.empty((total, small.pages.shape[1]), dtype=torch.uint8, device=DEV)
        pages[off:] = small.pages
        refs = torch.ones(total, dtype=torch.int32, device=DEV)
        refs[off:] = small.refs
        big = KVCache(plan, pages, torch.where(small.page_table >= 0, small.page_table + off, small.page_table), small.lengths.clone(), refs, 2, 64)
        mass = torch.empty((5, 2, wide), device=DEV)
        for count in (1, 12):
            gen = torch.Generator(device=DEV)
            gen.manual_seed(count)
            q = torch.randn((2 * count, 8, 128), generator=gen, device=DEV).to(torch.bfloat16)
            cu = [0, count, 2 * count]
            outs = [c.shared_attention(q, ints([3, 4]), ints(cu), None, count, max_prefix=1 << 27) for c in (small, big)]
            assert torch.equal(*outs)
            start = torch.rand((5, 2, narrow), generator=gen, device=DEV)
            mass[:, :, :narrow] = start
            want, tol = wanted(small, q, [3, 4], cu, start, 0.5, start)
            big.attention_mass(q, mass, ints([3, 4]), ints(cu), count, decay=0.5)
            assert bool(((mass[:, :, :narrow].double() - want).abs() <= tol).all())
        start = mass[:, :, :narrow].clone()
        results = [c.evict(m, 300, ints([4, 3]), recent=20, first=4) for c, m in ((small, start), (big, mass))]
        assert all(torch.equal(a, b) for a, b in zip(*results)) and results[0][0].eq(0).all()
        assert torch.equal(start, mass[:, :, :narrow])
        rows = [c.read(ints([3, 4]), ints([0, 300, 600]), 600) for c in (small, big)]
        assert all(torch.equal(a, b) for a, b in zip(*rows))


@pytest.mark.parametrize("asym,d,page", [(False, 128, 16), (True, 96, 64)])
def test_answers_to_a_document(asym, d, page):
    gbs_build.build()
    gen = torch.Generator(device=DEV)
    gen.manual_seed(7)
    new = lambda n, h: torch.randn((n, h, d), generator=gen, device=DEV).to(torch.bfloat16)  # noqa: E731
    with Plan(d, 128, 1, 4, 128, 0.9, asymmetric=asym) as plan:
        document, answers, keep = 700, 5, 150
        cache = KVCache.create(plan, 200, 2, page, 1 + answers, 60, DEV)
        mass = torch.full((1 + answers, 2, 1000), float("nan"), device=DEV)          # nothing of it is read before it was written
        # the document: its tokens, its attention, and what its last 32 tokens look back at
        seq, cu = ints([0]), ints([0, document])
        assert cache.extend(seq, ints([document])).item() == 0
        cache.append(new(document, 2), new(document, 2), seq, cu)
        q = new(document, 8) * 2
        out = cache.attention(q, seq, cu, document)
        want, tol = kv_util.attention(cache, q, [0], [0, document], few=False)
        assert bool(((out.double() - want).abs() <= tol).all())
        last = q[-32:].contiguous()
        expect, off = wanted(cache, last, [0], [0, 32], None, 0.0, mass)
        cache.attention_mass(last, mass, seq, ints([0, 32]), 32, decay=0.0)
        n = slice(0, document)
        assert bool(((mass[0, :, n].double() - expect[0, :, n]).abs() <= off[0, :, n]).all())
        # answers start from it, with what is known of its tokens
        forks = ints(range(1, 1 + answers))
        assert cache.fork(ints([0] * answers), forks).eq(0).all()
        mass[1:] = mass[0]
        lengths = [document] * answers
        for step in range(12):
            counts = [1] * answers if step % 4 else [3, 1, 2, 20, 1]
            cu_l = [0]
            for c in counts:
                cu_l.append(cu_l[-1] + c)
            total, cu = cu_l[-1], ints(cu_l)
            assert cache.extend(forks, ints(counts)).eq(0).all()
            cache.append(new(total, 2), new(total, 2), forks, cu)
            lengths = [a + c for a, c in zip(lengths, counts)]
            q = new(total, 8) * 2
            for prefix in (0, 1 << 27):                         # as the call judges itself, and shared in any case
                out = cache.shared_attention(q, forks, cu, None, max(counts), max_own=400, max_prefix=prefix)
                want, tol = kv_util.attention(cache, q, list(range(1, 1 + answers)), cu_l, few=False)
                assert bool(((out.double() - want).abs() <= tol).all()), step
            expect, off = wanted(cache, q, list(range(1, 1 + answers)), cu_l, mass.clone(), 0.9, mass)
            cache.attention_mass(q, mass, forks, cu, max(counts), decay=0.9)
            for i, a in enumerate(lengths):
                assert bool(((mass[1 + i, :, :a].double() - expect[1 + i, :, :a]).abs() <= off[1 + i, :, :a]).all()), (step, i)
            if step in (5, 10):                                 # the answers' copies are cut down; the document stays
                before = [kv_util.rows_of(cache, 1 + i) for i in range(answers)]
                w = mass.cpu().numpy()
                status, kept = cache.evict(mass, keep, forks, recent=20, first=4)
                assert status.eq(0).all()
                for i, a in enumerate(lengths):
                    for h in range(2):
                        p = stay(w[1 + i, h, :a], a, keep, 20, 4)
                        assert kept[i, h].tolist() == p
                        assert torch.equal(mass[1 + i, h, :keep].cpu(), torch.from_numpy(w[1 + i, h, p]))
                        k, v = kv_util.rows_of(cache, 1 + i)
                        assert torch.equal(k[h], before[i][0][h][p]) and torch.equal(v[h], before[i][1][h][p])
                lengths = [keep] * answers
            assert cache.lengths.tolist() == [document] + lengths
        held = sum(-(-a // page) for a in [document] + lengths)
        assert cache.refs.sum() == held and plan.device_status() == 0
        cache.free(ints(range(1 + answers)))
        assert cache.refs.eq(0).all()
