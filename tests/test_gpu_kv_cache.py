"""The paged KV cache on the GPU: rows written and read back, the pool's bookkeeping, and attention over it, against plain
implementations in 64 bits (kv_util)."""
import random

import numpy as np
import pytest
import torch

import kv_util
from kv_util import DEV, Model, filled
from paper_2504_13989_b200 import GbsError, KVCache, Plan, binding
from paper_2504_13989_b200 import build as gbs_build
from parity_util import TIE_WINDOW

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    gbs_build.build()


def plan_of(d=128, asym=False, alpha=0.9, group=128):
    return Plan(d, 128, 1, 4, group, alpha, asymmetric=asym)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def cu_of(counts):
    return np.concatenate([[0], np.cumsum(counts)]).tolist()


# ----------------------------------------------------------------------------------------------
# rows
# ----------------------------------------------------------------------------------------------
def check_rows(cache, x, pos, which):
    """The codes and scales of rows x [tokens, heads, d] at positions pos = [(sequence, position), ..]."""
    d, alpha, asym = cache.plan.info.d, float(np.float32(cache.plan.info.alpha)), bool(cache.plan.info.asymmetric)
    want = torch.zeros(x.shape[:2] + (128,), dtype=torch.float64, device=DEV)
    want[..., :d] = x.double()
    want = want @ kv_util.h128() / 128 ** 0.5
    got_q, got_s = [], []
    ps, sf = cache.page_size, 2 if asym else 1
    pages = cache.pages.view(cache.pages.shape[0], cache.n_kv_heads, -1)
    for s, p in pos:
        b = pages[int(cache.page_table[s, p // ps])]
        at = which * ps * 64 + (p % ps) * 64
        c = b[:, at:at + 64].to(torch.int16)
        got_q.append(torch.stack([c & 15, c >> 4], -1).flatten(-2))
        at = ps * 128 + (which * ps + p % ps) * 4 * sf
        got_s.append(b[:, at:at + 4 * sf].contiguous().view(torch.float32).double())
    q, s = torch.stack(got_q).double(), torch.stack(got_s)
    if asym:
        lo, hi = alpha * want.amin(-1), alpha * want.amax(-1)
        delta = (hi - lo) / 15
        # seven stages of additions round the rotated row by up to 7 2^-24 of the sum of its |x| / sqrt(128), lo and hi three times more
        err = 8 * 2.0 ** -24 * x.double().abs().sum(-1) / 128 ** 0.5 + 2.0 ** -22 * (lo.abs() + hi.abs())
        assert bool(((s[..., 0] - delta).abs() <= 2 * err / 15 + 2.0 ** -22 * delta).all()) and bool(((s[..., 1] - lo).abs() <= err).all())
        t = torch.where(delta[..., None] > 0, (want - lo[..., None]) / delta[..., None], 0.0)
        ref = t.round().clamp(0, 15)
    else:
        q = q - 16 * (q > 7)
        delta = alpha * want.abs().amax(-1) / 7
        assert bool(((s[..., 0] - delta).abs() <= 1e-6 * delta).all())
        t = torch.where(delta[..., None] > 0, want / delta[..., None], 0.0)
        ref = t.round().clamp(-7, 7)
    off = q != ref
    # Rows of few distinct values can lie on ties: 80 ones rotate to -16, 0, 16, 48 and 80 (times 1 / sqrt(128)), and the asymmetric quantizer
    # puts each 0 at 15 * 16 / 96 = 2.5 exactly (alpha shrinks lo and the span alike); 32 bits then fall on either side.  Such codes do not count.
    tie = ((t - t.floor()) - 0.5).abs() < 1e-12
    assert bool(((q - ref).abs() <= 1).all()) and float((off & ~tie).double().mean()) <= 1e-4
    assert bool(((t[off] - t[off].floor() - 0.5).abs() < 4 * TIE_WINDOW).all())


@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("d,heads,page", [(128, 8, 64), (80, 3, 16), (8, 1, 32), (96, 2, 128), (128, 1, 16)])
def test_append_and_read(d, heads, page, asym):
    counts, have = [1, 37, 0, 130, 16, 5], [0, 3, 9, 64, 15, 200]
    gen = torch.Generator(device=DEV)
    gen.manual_seed(d + heads)
    with plan_of(d, asym) as plan:
        cache = filled(plan, [a + b for a, b in zip(counts, have)], heads, page, seed=1)
        order = [3, 0, 5, 1, 2, 4]
        cu = cu_of([counts[s] for s in order])
        total = cu[-1]
        k = (torch.randn((total, heads, d), generator=gen, device=DEV).pow(3)).to(torch.bfloat16)
        v = torch.randn((total, heads, d), generator=gen, device=DEV).to(torch.bfloat16)
        k[7] = 0
        v[3, 0] = 1.0
        before = cache.pages.clone()
        cache.append(k, v, ints(order), ints(cu))
        pos = [(s, have[s] + j) for s in order for j in range(counts[s])]
        check_rows(cache, k, pos, 0)
        check_rows(cache, v, pos, 1)
        # nothing else of the pool changes
        mine = torch.zeros_like(before, dtype=torch.bool).view(before.shape[0], heads, -1)
        sf = 2 if asym else 1
        for s, p in pos:
            b = mine[int(cache.page_table[s, p // page])]
            for which in range(2):
                b[:, which * page * 64 + (p % page) * 64:][:, :64] = True
                b[:, page * 128 + (which * page + p % page) * 4 * sf:][:, :4 * sf] = True
        assert bool(((cache.pages == before) | mine.view_as(before)).all())

        out = [torch.full((total + 2, heads, d), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        cache.read(ints(order), ints(cu), out=tuple(out))
        torch.cuda.synchronize()
        for which in range(2):
            want = []
            for s in order:
                y = kv_util.rows_of(cache, s)[which].transpose(0, 1)[have[s]:]
                want.append((y @ kv_util.h128() / 128 ** 0.5)[..., :d])
            want = torch.cat(want)
            # the exact sum of 128 codes (at most 15 each), times a factor of two roundings; lo sqrt(128) comes with one more of each
            bound = 2.0 ** -8 * want.abs() + 2.0 ** -21 * want.abs().amax(-1, keepdim=True) + 2.0 ** -20 * 128 ** 0.5 * 8
            assert bool(((out[which][:total].double() - want).abs() <= bound).all())
            assert bool((out[which][total:] == 7.0).all())


def test_append_matches_rotate_quantize_and_takes_strides():
    """The same codes as the framework's own rows, from a packed [tokens, 3, heads, d] projection, on another stream."""
    with plan_of(128) as plan:
        cache = filled(plan, [50, 3], 4, 16)
        gen = torch.Generator(device=DEV)
        gen.manual_seed(5)
        qkv = torch.randn((53, 3, 4, 128), generator=gen, device=DEV).to(torch.bfloat16)
        cu = ints([0, 50, 53])
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        cache.append(qkv[:, 1], qkv[:, 2], None, cu, stream=side)
        side.synchronize()
        for which in (1, 2):
            codes, scales, _ = plan.rotate_quantize(qkv[:, which].contiguous())
            y = plan.dequantize(codes, scales).view(53, 4, 128).double()
            got = torch.cat([kv_util.rows_of(cache, s)[which - 1].transpose(0, 1) for s in (0, 1)])
            assert float(((got - y).abs() > 1e-5).double().mean()) <= 1e-4


@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("size", [2.0 ** -126, 2.0 ** -100, 2.0 ** 100, 2.0 ** 116])
def test_rows_near_the_ends_of_the_range(size, asym):
    with plan_of(128, asym, alpha=1.0) as plan:
        cache = filled(plan, [40], 2, 16)
        gen = torch.Generator(device=DEV)
        gen.manual_seed(9)
        k = (torch.randn((40, 2, 128), generator=gen, device=DEV).clamp(-3, 3) * size).to(torch.bfloat16)
        cache.append(k, k, None, ints([0, 40]))
        y = k.double() @ kv_util.h128() / 128 ** 0.5
        got = kv_util.rows_of(cache, 0)[1].transpose(0, 1)
        span = y.amax(-1, keepdim=True) - y.amin(-1, keepdim=True) if asym else y.abs().amax(-1, keepdim=True)
        # half a step, and what the smallest numbers lose of the scales (2^-150 each, times 15 codes)
        step = span / (15 if asym else 7)
        assert bool(((got - y).abs() <= 0.5001 * step + 32 * 2.0 ** -149).all())


def test_bad_numbers_on_the_device_leave_tokens_out():
    with plan_of(128) as plan:
        cache = filled(plan, [20, 30, 5], 2, 16)
        cache.page_table[1, 0] = 10 ** 6
        cache.page_table[1, 1] = -5
        before = cache.pages.clone()
        x = torch.ones((4, 2, 128), dtype=torch.bfloat16, device=DEV)
        cache.append(x, x, ints([1, 7, -1, 2 ** 31 - 1]))                  # a bad page, and sequences out of range
        many = torch.ones((9, 2, 128), dtype=torch.bfloat16, device=DEV)
        cache.append(many[:4], many[:4], ints([2]), ints([0, 0]))           # rows behind the last item
        assert torch.equal(cache.pages, before)
        k, v = cache.read(ints([1, 7, -1, 2 ** 31 - 1]))
        assert not k.any() and not v.any()
        k, v = cache.read(ints([2]), ints([0, 9]), 9)                       # nine tokens of a sequence that has five
        assert not k[:4].any() and bool(k[4:].any())
        cache.append(many, many, ints([2]), ints([0, 9]))
        got = kv_util.rows_of(cache, 2)[0]
        # a row of ones becomes sqrt(128) = 11.31 in its first coordinate, clipped to 0.9 of it
        assert got.shape[1] == 5 and bool(((got[..., 0] - 0.9 * 128 ** 0.5).abs() < 1e-5).all())


# ----------------------------------------------------------------------------------------------
# bookkeeping
# ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("n_pages,page,n_seqs,max_pages,heads", [(40, 16, 12, 6, 2), (9000, 32, 300, 40, 1), (7, 128, 5, 3, 3), (64, 64, 33, 4, 1)])
def test_bookkeeping(n_pages, page, n_seqs, max_pages, heads, asym):
    rng = random.Random(n_pages)
    with plan_of(128, asym) as plan:
        cache = KVCache.create(plan, n_pages, heads, page, n_seqs, max_pages, DEV)
        gen = torch.Generator(device=DEV)
        gen.manual_seed(1)
        cache.pages.random_(0, 256, generator=gen)
        model = Model(n_pages, page, n_seqs, max_pages)
        for step in range(30):
            n = rng.randrange(1, n_seqs + 3)
            what = rng.choice(["extend", "extend", "fork", "free"])
            if what == "extend":
                seqs = [rng.randrange(-1, n_seqs + 1) for _ in range(n)]
                counts = [rng.choice([0, 1, 1, page, rng.randrange(-1, 2 * page + 2), max_pages * page]) for _ in range(n)]
                assert cache.extend(ints(seqs), ints(counts)).tolist() == model.extend(seqs, counts)
            elif what == "fork":
                src, dst = ([rng.randrange(-1, n_seqs + 1) for _ in range(n)] for _ in range(2))
                before = cache.pages.clone()
                model.copies = []
                assert cache.fork(ints(src), ints(dst)).tolist() == model.fork(src, dst)
                want = before.view(n_pages, heads, -1)
                old, sf = want.clone(), 2 if asym else 1
                for a, b, tail in model.copies:
                    for at, size in ((0, 64), (page * 64, 64), (page * 128, 4 * sf), (page * (128 + 4 * sf), 4 * sf)):
                        want[b, :, at:at + tail * size] = old[a, :, at:at + tail * size]
                assert torch.equal(cache.pages, before)
            else:
                seqs = [rng.randrange(-1, n_seqs + 1) for _ in range(n)]
                cache.free(ints(seqs))
                model.free(seqs)
            model.check(cache)


def test_extend_every_sequence_by_a_token_and_more_items_than_a_block():
    with plan_of(128) as plan:
        cache = KVCache.create(plan, 5000, 1, 16, 4000, 3, DEV)
        model = Model(5000, 16, 4000, 3)
        for _ in range(3):
            assert cache.extend().tolist() == model.extend(list(range(4000)), [1] * 4000)
            assert cache.extend(None, ints([7] * 3000)).tolist() == model.extend(list(range(3000)), [7] * 3000)
            model.check(cache)
        src, dst = [s % 900 for s in range(1000)], list(range(3000, 4000))
        cache.free(ints(dst))
        model.free(dst)
        assert cache.fork(ints(src), ints(dst)).tolist() == model.fork(src, dst)
        model.check(cache)
        with pytest.raises(GbsError):
            cache.extend(torch.zeros(binding.GBS_KV_MAX_ITEMS + 1, dtype=torch.int32, device=DEV))


@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("n_pages,into_pages,heads,page", [(50, 50, 2, 16), (50, 31, 1, 32), (9000, 20000, 1, 16), (12, 12, 40, 128)])
def test_compact(n_pages, into_pages, heads, page, asym):
    rng = random.Random(into_pages)
    n_seqs = max(4, n_pages // 20)
    with plan_of(128, asym) as plan:
        cache = KVCache.create(plan, n_pages, heads, page, n_seqs, 30, DEV)
        gen = torch.Generator(device=DEV)
        gen.manual_seed(3)
        cache.pages.random_(0, 256, generator=gen)
        cache.extend(None, ints([rng.randrange(0, 12 * page) for _ in range(n_seqs)]))
        cache.free(ints([s for s in range(n_seqs) if s % 3 == 0]))
        cache.fork(ints([1]), ints([0]))
        into = KVCache.create(plan, into_pages, heads, page, n_seqs, 30, DEV)
        into.pages.fill_(9)
        into.lengths.fill_(5)
        into.refs.fill_(3)
        page_map = torch.full((n_pages,), 77, dtype=torch.int32, device=DEV)
        live = cache.compact(into, page_map)
        refs = cache.refs.tolist()
        used = [p for p, r in enumerate(refs) if r > 0]
        assert live.tolist() == [len(used)]
        new = {p: i for i, p in enumerate(used) if i < into_pages}
        assert page_map.tolist() == [new.get(p, -1) for p in range(n_pages)]
        assert into.refs.tolist() == ([refs[p] for p in used] + [0] * into_pages)[:into_pages]
        moved = used[:into_pages]
        assert torch.equal(into.pages[:len(moved)], cache.pages[moved]) and bool((into.pages[len(moved):] == 9).all())
        assert torch.equal(into.lengths, cache.lengths)
        old, lengths = cache.page_table.tolist(), cache.lengths.tolist()
        assert into.page_table.tolist() == [[new.get(p, -1) if j < -(-lengths[s] // page) else -1 for j, p in enumerate(row)] for s, row in enumerate(old)]


# ----------------------------------------------------------------------------------------------
# attention
# ----------------------------------------------------------------------------------------------
def check_attention(cache, seqs, counts, heads, q_scale=3.0, seed=0, **kw):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    d, total = cache.plan.info.d, sum(counts)
    q = (torch.randn((total, heads, d), generator=gen, device=DEV) * q_scale * (128 / d) ** 0.5).to(torch.bfloat16)
    cu = cu_of(counts)
    most = max(1, max(counts))
    got = cache.attention(q, ints(seqs), ints(cu), most, **kw)
    few = most * (heads // cache.n_kv_heads) <= 16
    want, tol = kv_util.attention(cache, q, seqs, cu, few=few, **kw)
    off = (got.double() - want).abs()
    assert bool((off <= tol).all()), (float((off - tol).max()), float((off / tol.clamp(min=1e-30)).max()))
    return q, got


HEADS = [(32, 8, 128), (8, 8, 80), (8, 1, 128), (16, 1, 128), (14, 2, 64), (5, 5, 8), (40, 2, 96), (1, 1, 128)]


@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("heads,kv_heads,d", HEADS)
def test_single_tokens(heads, kv_heads, d, page, asym):
    lengths = [1, 15, 16, 17, 63, 129, 0, 300, 1000]
    with plan_of(d, asym) as plan:
        cache = filled(plan, lengths, kv_heads, page, seed=heads)
        seqs = [8, 1, 0, 2, 6, 3, 4, 5, 7]
        check_attention(cache, seqs, [1] * 9, heads)
        check_attention(cache, seqs, [1] * 9, heads, window=20, max_len=1000, scale=0.05)


@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("heads,kv_heads,d", HEADS)
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 33), (False, 33)])
def test_few_tokens(heads, kv_heads, d, causal, window, asym):
    lengths = [3, 40, 200, 2, 0, 513, 1]
    counts = [3, 2, 4, 4, 1, 0, 1]                          # the fourth asks for more tokens than it has
    with plan_of(d, asym) as plan:
        cache = filled(plan, lengths, kv_heads, 32, seed=heads)
        check_attention(cache, list(range(7)), counts, heads, causal=causal, window=window)


@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("heads,kv_heads,d,page", [(32, 8, 128, 16), (8, 8, 80, 64), (14, 2, 64, 128), (4, 1, 128, 32)])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 100), (False, 100)])
def test_prompts(heads, kv_heads, d, page, causal, window, asym):
    lengths = [130, 1, 700, 0, 64, 333, 20]
    counts = [130, 1, 129, 2, 17, 333, 31]                  # whole prompts, chunks behind a cache, and more tokens than there are
    with plan_of(d, asym) as plan:
        cache = filled(plan, lengths, kv_heads, page, seed=page)
        check_attention(cache, [4, 0, 2, 1, 3, 5, 6], [counts[i] for i in [4, 0, 2, 1, 3, 5, 6]], heads, causal=causal, window=window)


@pytest.mark.parametrize("counts", [[1], [1, 1, 1], [2, 4], [100]])
def test_long_cache(counts):
    """Few rows and many tokens: the long axis is split and joined."""
    with plan_of(128) as plan:
        lengths = [40000, 3, 20011][:len(counts)]
        lengths[-1] = max(lengths[-1], counts[-1])
        cache = filled(plan, lengths, 2, 64, seed=4, scale=0.3)
        check_attention(cache, list(range(len(counts))), counts, 8)
        check_attention(cache, list(range(len(counts))), counts, 8, max_len=40000, window=9000)


def test_scores_that_differ_by_much():
    """The largest score comes late, or first, and is far above the rest; values of very different sizes."""
    with plan_of(128, alpha=1.0) as plan:
        gen = torch.Generator(device=DEV)
        gen.manual_seed(11)
        for at in (0, 700, 1499):
            cache = filled(plan, [1500], 1, 16, seed=8, scale=0.05)
            k = torch.randn((1500, 1, 128), generator=gen, device=DEV) * 0.05
            k[at] = 3.0
            k[700:] *= 30.0
            v = torch.randn((1500, 1, 128), generator=gen, device=DEV) * torch.logspace(-3, 3, 1500, device=DEV)[:, None, None]
            cache.append(k.to(torch.bfloat16), v.to(torch.bfloat16), None, ints([0, 1500]))
            for counts in ([1], [3], [60]):
                check_attention(cache, [0], counts, 4, q_scale=4.0)


def test_rows_of_other_tokens_stay_and_nan_stays_in_its_row():
    with plan_of(128) as plan:
        cache = filled(plan, [90, 50], 2, 16)
        for counts in ([1, 2], [40, 30]):
            total = sum(counts)
            q = torch.randn((total + 3, 8, 128), device=DEV).to(torch.bfloat16)
            out = torch.full((total + 3, 8, 128), 7.0, dtype=torch.bfloat16, device=DEV)
            cu = ints(cu_of(counts))
            cache.attention(q, ints([1, 0]), cu, max(counts), out=out)
            assert bool((out[total:] == 7.0).all()) and bool(torch.isfinite(out.float()).all())
            bad = q.clone()
            bad[1, 3, 5] = float("nan")
            bad[total - 1, 0, 0] = float("inf")
            got = cache.attention(bad[:total], ints([1, 0]), cu, max(counts))
            assert bool(torch.isnan(got[1, 3]).all()) and bool(torch.isnan(got[total - 1, 0]).all())
            same = torch.ones((total, 8), dtype=torch.bool, device=DEV)
            same[1, 3] = same[total - 1, 0] = False
            assert torch.equal(got[same], out[:total][same])


def test_bad_pages_and_sequences():
    """Tokens without a page are not seen; items without a sequence become 0."""
    with plan_of(128) as plan:
        cache = filled(plan, [100, 40], 2, 16)
        good = KVCache(plan, cache.pages, cache.page_table.clone(), ints([80, 40]), cache.refs, 2, 16)
        for rows in (1, 30):
            q = torch.randn((rows, 4, 128), device=DEV).to(torch.bfloat16)
            cu = ints([0, rows])
            want = good.attention(q, ints([0]), cu, rows, causal=False)
            cache.page_table[0, 5] = 10 ** 7
            cache.page_table[0, 6] = -1
            got = cache.attention(q, ints([0]), cu, rows, causal=False)
            assert float((got.double() - want.double()).abs().max()) <= 2.0 ** -7 * float(want.abs().max())
            for s in (2, -1, 2 ** 31 - 1):
                assert not cache.attention(q, ints([s]), cu, rows).any()


def test_strides_streams_and_graphs():
    with plan_of(96) as plan:
        cache = filled(plan, [500, 77, 130], 4, 32)
        for counts in ([1, 1, 1], [60, 77, 1]):
            total, most, cu = sum(counts), max(counts), ints(cu_of(counts))
            qkv = torch.randn((total, 24, 96), device=DEV).to(torch.bfloat16)
            q = qkv[:, 4:12]
            want = cache.attention(q.contiguous(), None, cu, most)
            out = torch.zeros((8, total, 96), dtype=torch.bfloat16, device=DEV).transpose(0, 1)
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            cache.attention(q, None, cu, most, out=out, stream=side)
            side.synchronize()
            assert torch.equal(out, want)
            # captured and replayed, with other contents
            g = torch.cuda.CUDAGraph()
            q2 = q.contiguous()
            with torch.cuda.graph(g):
                got = cache.attention(q2, None, cu, most)
            for _ in range(3):
                q2.copy_(torch.randn_like(q2))
                g.replay()
                want2 = cache.attention(q2, None, cu, most)
                assert torch.equal(got, want2)


def test_refusals_of_the_binding():
    with plan_of(128) as plan, Plan(128, 128, 1, 3, 128, 1.0) as three:
        cache = filled(plan, [20], 2, 16)
        q = torch.randn((1, 4, 128), device=DEV).to(torch.bfloat16)
        with pytest.raises(GbsError):
            KVCache.create(three, 4, 2, 16, 2, 2, DEV)
        for bad in (q.float(), q.half()):
            with pytest.raises(TypeError):
                cache.attention(bad)
        for bad in (q[0], q[..., :64], q.cpu(), q.transpose(1, 2)):
            with pytest.raises(ValueError):
                cache.attention(bad)
        with pytest.raises(GbsError):
            cache.attention(q[:, :3])                       # three heads over two
        with pytest.raises(ValueError):
            cache.append(q[:, :2], q[:, :2], ints([0, 0, 0])[:2], ints([0, 1]))
        with pytest.raises(ValueError):
            cache.append(q[:, :2], q[:, :2].repeat(2, 1, 1))
        with pytest.raises((TypeError, ValueError)):
            cache.append(q[:, :2], q[:, :2], torch.zeros(1, dtype=torch.int64, device=DEV))
        with pytest.raises(ValueError):
            cache.read(None, ints([0, 3]))
        with pytest.raises(ValueError):
            KVCache(plan, cache.pages[:, :-16], cache.page_table, cache.lengths, cache.refs, 2, 16)
        with pytest.raises(ValueError):
            KVCache(plan, cache.pages, cache.page_table, cache.lengths[:0], cache.refs, 2, 16)


# ----------------------------------------------------------------------------------------------
# a run of them together
# ----------------------------------------------------------------------------------------------
def test_a_serving_loop():
    """Prompts, decoding steps, a fork, an end and a move to another pool, with the outputs of every step checked; the step in a graph."""
    heads, kvh, d, page = 8, 2, 80, 16
    with plan_of(d) as plan:
        cache = KVCache.create(plan, 60, kvh, page, 6, 20, DEV)
        gen = torch.Generator(device=DEV)
        gen.manual_seed(2)
        rnd = lambda n, h: torch.randn((n, h, d), generator=gen, device=DEV).to(torch.bfloat16)  # noqa: E731
        counts, seqs = [33, 100, 7], [0, 2, 5]
        assert cache.extend(ints(seqs), ints(counts)).tolist() == [0, 0, 0]
        cache.append(rnd(140, kvh), rnd(140, kvh), ints(seqs), ints(cu_of(counts)))
        check_attention(cache, seqs, counts, heads)
        assert cache.fork(ints([2, 2]), ints([1, 3])).tolist() == [0, 0]
        seqs = [0, 1, 2, 3, 5]
        s = ints(seqs)
        for step in range(20):
            assert not cache.extend(s).any()
            cache.append(rnd(5, kvh), rnd(5, kvh), s)
            check_attention(cache, seqs, [1] * 5, heads, seed=step)
        cache.free(ints([2, 0]))
        into = KVCache.create(plan, 30, kvh, page, 6, 20, DEV)
        live = int(cache.compact(into))
        assert live == int((cache.refs > 0).sum()) <= 30
        q = rnd(3, heads)
        s = ints([1, 3, 5])
        assert torch.equal(cache.attention(q, s), into.attention(q, s))
        # a decoding step as one graph
        k, v = rnd(3, kvh), rnd(3, kvh)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            into.extend(s)
            into.append(k, v, s)
            got = into.attention(q, s)
        for step in range(18):
            k.copy_(rnd(3, kvh))
            g.replay()
            want, tol = kv_util.attention(into, q, [1, 3, 5], [0, 1, 2, 3])
            assert bool(((got.double() - want).abs() <= tol).all())
        assert into.lengths[[1, 3, 5]].tolist() == (cache.lengths[[1, 3, 5]] + 18).tolist()


def test_native_and_python_paths_agree():
    """The regular calls of _native.so against the functions that they stand in front of; calls after the plan is closed are refused."""
    def python(name):
        return getattr(KVCache, name).__wrapped__
    # tokens that were given room and not written hold what the pool held: numbers that are none, where one is seen
    same = lambda x, y: torch.allclose(x, y, rtol=0, atol=0, equal_nan=True)  # noqa: E731
    gen = torch.Generator(device=DEV)
    gen.manual_seed(6)
    plan = plan_of(96)
    a, b = (filled(plan, [40, 3, 0, 100], 2, 16, seed=2, spare=40) for _ in range(2))
    seqs, counts = ints([3, 2, 0]), ints([2, 5, 1])
    cu = ints([0, 2, 7, 8])
    for s, c in ((seqs, counts), (None, None), (seqs, None)):
        assert torch.equal(a.extend(s, c), python("extend")(b, s, c))
    a.free(seqs=ints([1])), python("free")(b, ints([1]))
    assert torch.equal(a.fork(ints([3]), dst=ints([1])), python("fork")(b, ints([3]), ints([1])))
    k, v = (torch.randn((8, 2, 96), generator=gen, device=DEV).to(torch.bfloat16) for _ in range(2))
    assert a.append(k, v, seqs, cu_tokens=cu) is None
    python("append")(b, k, v, seqs, cu)
    for x in ("pages", "page_table", "lengths", "refs"):
        x, y = getattr(a, x), getattr(b, x)
        assert torch.equal(x, y)
    for x, y in zip(a.read(seqs, cu, 8), python("read")(b, seqs, cu, 8)):
        assert torch.equal(x, y)
    q = torch.randn((8, 6, 96), generator=gen, device=DEV).to(torch.bfloat16)
    want = python("attention")(b, q, seqs, cu, 5, causal=False, window=30, scale=0.1, max_len=64)
    assert same(a.attention(q, seqs, cu, 5, causal=False, window=30, scale=0.1, max_len=64), want)
    out = torch.empty_like(q)
    assert a.attention(q, seqs, cu, 5, False, 30, 0.1, 64, out) is out and same(out, want)
    wide = torch.zeros((8, 12, 96), dtype=torch.bfloat16, device=DEV)
    wide[:, :6] = q
    assert same(a.attention(wide[:, :6], seqs, cu, 5, causal=False, window=30, scale=0.1, max_len=64), want)
    with pytest.raises(GbsError):
        a.attention(q, seqs, cu, 0)
    into = [KVCache.create(plan, 60, 2, 16, 4, a.page_table.shape[1], DEV) for _ in range(2)]
    maps = [torch.empty(a.pages.shape[0], dtype=torch.int32, device=DEV) for _ in range(2)]
    assert torch.equal(a.compact(into[0], page_map=maps[0]), python("compact")(b, into[1], maps[1])) and torch.equal(maps[0], maps[1])
    assert torch.equal(a.compact(into[0]), b.compact(into[1], maps[1])) and torch.equal(into[0].page_table, into[1].page_table)
    with pytest.raises(GbsError):
        a.compact(a)
    plan.close()
    with pytest.raises(GbsError):
        a.attention(q, seqs, cu, 5)
    with pytest.raises(GbsError):
        a.extend()


# ----------------------------------------------------------------------------------------------
# calls at the edges of what is allowed
# ----------------------------------------------------------------------------------------------
def test_rows_before_the_first_item_are_not_written():
    with plan_of(128) as plan:
        cache = filled(plan, [20, 9], 2, 16)
        before = cache.pages.clone()
        x = torch.ones((6, 2, 128), dtype=torch.bfloat16, device=DEV)
        cache.append(x, x, None, ints([6, 6, 6]))
        assert torch.equal(cache.pages, before)
        cache.append(x, x, None, ints([4, 6, 6]))                           # the last two tokens of sequence 0
        assert torch.equal(kv_util.rows_of(cache, 0, 18)[0], kv_util.rows_of(KVCache(plan, before, cache.page_table, cache.lengths, cache.refs, 2, 16), 0, 18)[0])
        assert not torch.equal(cache.pages, before)


@pytest.mark.parametrize("counts", [[1, 1], [3, 3], [40, 70]])
def test_the_widest_window_and_items_with_more_tokens_than_their_sequence(counts):
    with plan_of(128) as plan:
        cache = filled(plan, [130, 33], 2, 32)
        for window in (2 ** 31 - 1, 2 ** 30, 2 ** 27):
            for causal in (True, False):
                check_attention(cache, [0, 1], counts, 4, causal=causal, window=window)


@pytest.mark.parametrize("counts", [[1, 1, 1], [30, 1, 64]])
def test_one_sequence_read_by_several_items(counts):
    with plan_of(80) as plan:
        cache = filled(plan, [200, 90], 2, 16)
        check_attention(cache, [0, 0, 1], counts, 8)


def test_two_graphs_on_two_streams_and_calls_between_them():
    """Two captured steps on one pool, replayed at the same time; each has a workspace of its own."""
    with plan_of(128) as plan:
        cache = filled(plan, [5000, 900, 40], 4, 64)
        gen = torch.Generator(device=DEV)
        gen.manual_seed(3)
        work = []
        for counts in ([1, 1, 1], [100, 33, 40]):
            cu, most = ints(cu_of(counts)), max(counts)
            q = torch.randn((sum(counts), 16, 128), generator=gen, device=DEV).to(torch.bfloat16)
            want = cache.attention(q, None, cu, most)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                out = cache.attention(q, None, cu, most)
            work.append((g, out, want, torch.cuda.Stream(), q, cu, most))
        torch.cuda.synchronize()
        for _ in range(5):
            for g, out, _, s, _, _, _ in work:
                out.zero_()
            torch.cuda.synchronize()
            for g, _, _, s, _, _, _ in work:
                with torch.cuda.stream(s):
                    g.replay()
            eager = [cache.attention(q, None, cu, most) for _, _, _, _, q, cu, most in work]
            torch.cuda.synchronize()
            for (_, out, want, *_), e in zip(work, eager):
                assert torch.equal(out, want) and torch.equal(e, want)
        assert plan.device_status() == 0


def test_a_whole_step_is_captured():
    """extend, append and attention of a step in one graph: every replay adds a token to each sequence."""
    with plan_of(128) as plan:
        n, steps = 5, 40
        a, b = (KVCache.create(plan, 40, 2, 16, n, 8, DEV) for _ in range(2))
        gen = torch.Generator(device=DEV)
        gen.manual_seed(9)
        x = torch.randn((steps, 3, n, 8, 128), generator=gen, device=DEV).to(torch.bfloat16)
        q, k, v = torch.zeros_like(x[0, 0]), torch.zeros_like(x[0, 0, :, :2]).contiguous(), torch.zeros_like(x[0, 0, :, :2]).contiguous()

        def step(cache):
            status = cache.extend()
            cache.append(k, v)
            return status, cache.attention(q)
        step(a)                                                             # what a first call sets up
        for t in (a.lengths, a.refs):
            t.zero_()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            status, got = step(a)
        for t in (a.lengths, a.refs):
            t.zero_()
        for i in range(steps):
            q.copy_(x[i, 0]), k.copy_(x[i, 1, :, :2]), v.copy_(x[i, 2, :, :2])
            g.replay()
            want_status, want = step(b)
            assert not status.any() and torch.equal(status, want_status) and torch.equal(got, want)
            assert a.lengths.tolist() == [i + 1] * n == b.lengths.tolist()


def test_without_max_tokens_every_row_is_answered():
    with plan_of(128) as plan:
        cache = filled(plan, [90, 50, 7], 2, 16)
        for counts in ([1, 1, 1], [2, 0, 3], [40, 30, 1]):
            q = torch.randn((sum(counts), 8, 128), device=DEV).to(torch.bfloat16)
            cu = ints(cu_of(counts))
            few = sum(counts) * 4 <= 16
            want, tol = kv_util.attention(cache, q, [0, 1, 2], cu_of(counts), few=few)
            python = binding._PYTHON_KV_METHODS["attention"](cache, q, None, cu)
            for got in (cache.attention(q, None, cu), cache.attention(q, None, cu, None), python):
                assert bool(((got.double() - want).abs() <= tol).all())


def test_more_refusals_of_the_binding():
    with plan_of(128) as plan:
        cache = filled(plan, [20], 2, 16)
        q = torch.randn((1, 4, 128), device=DEV).to(torch.bfloat16)
        with pytest.raises(GbsError):
            cache.attention(q, out=q)
        for name in ("max_tokens", "window", "max_len"):
            with pytest.raises(ValueError):
                cache.attention(q, **{name: 2 ** 32 + 1})
            with pytest.raises(GbsError):
                cache.attention(q, **{name: -1})
        other = plan._device
        plan._device = other + 1
        with pytest.raises(ValueError):
            KVCache(plan, cache.pages, cache.page_table, cache.lengths, cache.refs, 2, 16)
        plan._device = other
        want = cache.attention(q)
        cache.lengths = torch.zeros_like(cache.lengths)                     # a name, not the pool's tensor
        assert torch.equal(cache.attention(q), want)


@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("count", [1, 3, 60, 150])
def test_scales_that_are_no_numbers_reach_the_rows_that_see_them(count, asym):
    with plan_of(128, asym) as plan:
        for which, bad in ((0, float("nan")), (1, float("nan")), (1, float("inf"))):
            cache = filled(plan, [200], 2, 32)
            gen = torch.Generator(device=DEV)
            gen.manual_seed(count)
            q = torch.randn((count, 4, 128), generator=gen, device=DEV).to(torch.bfloat16)
            cu, few = ints([0, count]), 2 * count <= 16
            want, tol = kv_util.attention(cache, q, [0], [0, count], few=few)
            at = max(180, 200 - count // 2)                                 # this token's scale, of KV head 1
            sf = 2 if asym else 1
            block = cache.pages[cache.page_table[0, at // 32].long()].view(2, -1)[1]
            block[32 * 128:].view(torch.float32)[which * 32 * sf + (at % 32) * sf] = bad
            got = cache.attention(q, ints([0]), cu, count).double()
            sees = torch.zeros((count, 4), dtype=torch.bool, device=DEV)
            sees[torch.arange(200 - count, 200, device=DEV) >= at, 2:] = True
            assert bool(torch.isnan(got[sees]).all()) and bool(((got - want).abs() <= tol)[~sees].all())


@pytest.mark.parametrize("counts", [[1], [3], [300]])
def test_values_of_zero_and_of_many_sizes(counts):
    """Zero values first, then ever larger ones; the rows of a long prompt see some of them each.  Groups of 32 tokens have one size."""
    with plan_of(128, alpha=1.0) as plan:
        cache = filled(plan, [300], 2, 16, scale=0.1)
        gen = torch.Generator(device=DEV)
        gen.manual_seed(21)
        k = (torch.randn((300, 2, 128), generator=gen, device=DEV) * 0.1).to(torch.bfloat16)
        size = torch.tensor([0.0, 0.0, 2.0 ** -40, 2.0 ** -38, 0.0, 2.0 ** -20, 1.0, 2.0 ** 6, 2.0 ** 30, 0.0], device=DEV).repeat_interleave(32)[:300]
        v = (torch.randn((300, 2, 128), generator=gen, device=DEV) * size[:, None, None]).to(torch.bfloat16)
        for _ in range(2):
            cache.append(k, v, None, ints([0, 300]))
            check_attention(cache, [0], counts, 6)
            check_attention(cache, [0], counts, 6, window=40)
            v = v.flip(0).contiguous()                                      # the largest first


@pytest.mark.parametrize("asym", [False, True])
def test_a_negative_scale_and_windows_at_every_offset(asym):
    with plan_of(64, asym) as plan:
        cache = filled(plan, [260], 1, 16)
        for counts in ([2], [130]):
            check_attention(cache, [0], counts, 3, scale=-0.2)
            for window in (1, 2, 31, 32, 33, 64, 127, 128, 129):
                check_attention(cache, [0], counts, 3, window=window)


def test_prompts_of_every_length_around_a_tile():
    """One KV head with three query heads: rows that fill one tile of 128, both, or a little of the next block's."""
    with plan_of(128) as plan:
        for count in (6, 42, 43, 44, 85, 86, 87, 128, 171, 172):
            cache = filled(plan, [count, count + 1, count + 200], 1, 64, seed=count)
            check_attention(cache, [0, 1, 2], [count] * 3, 3)
