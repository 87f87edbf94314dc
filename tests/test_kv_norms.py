"""The attention over the paged KV cache by the norms of its rows (kv_norms): on the CPU that the bound lets the roundings through and no lost, repeated or
misplaced tokens; on the GPU every form of the call."""
import numpy as np
import pytest
import torch

import kv_norms
import kv_util


# ----------------------------------------------------------------------------------------------
# what the bound tells apart
# ----------------------------------------------------------------------------------------------
def cached(n, asym, gen, heads=2):
    """Rotated rows as the quantizer leaves them, and their middles."""
    y = torch.randn((heads, n, 128), generator=gen, dtype=torch.float64)
    if asym:
        lo, hi = 0.9 * y.amin(-1, keepdim=True), 0.9 * y.amax(-1, keepdim=True)
        delta = (hi - lo) / 15
        return ((y - lo) / delta).round().clamp(0, 15) * delta + lo, (lo + 8 * delta)[..., 0]
    delta = 0.9 * y.abs().amax(-1, keepdim=True) / 7
    return (y / delta).round().clamp(-7, 7) * delta, torch.zeros_like(y[..., 0])


def half(x):
    return x.half().double()


def kernel_like(x, k, km, v, vm, seen, scale, few):
    """The roundings that the bound counts, and no other error."""
    if few:
        m = x.abs().amax(-1, keepdim=True) / 32512
        s = torch.einsum("qhgd,hkd->qhgk", (x / m).round() * m, k)
    else:
        def rounded(y, mid):
            # a power of two for each row, as a group of 32 tokens has one; Delta c with Delta rounded is c' (1 + e)
            e = half(torch.full_like(mid, 1.2345)) / 1.2345
            return half((y - mid[..., None]) * e[..., None] + half(mid)[..., None])
        s = torch.einsum("qhgd,hkd->qhgk", half(x), rounded(k, km))
        v = rounded(v, vm)
    s = (s * scale).masked_fill(~seen[:, None, None], float("-inf"))
    w = torch.exp(s - s.amax(-1, keepdim=True)) * 64
    if few:
        o = torch.einsum("qhgk,hkd->qhgd", half(w), v - vm[..., None]) + torch.einsum("qhgk,hk->qhg", w, vm)[..., None]
    else:
        o = torch.einsum("qhgk,hkd->qhgd", half(w), v)
    o = o / w.sum(-1, keepdim=True)
    return o.to(torch.bfloat16).double()


CASES = [(1, 40000, 4, 0), (1, 1000, 1, 0), (3, 513, 4, 33), (129, 700, 4, 100), (333, 333, 4, 0), (64, 8000, 8, 0)]


@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("size", [0.5, 3.0])
@pytest.mark.parametrize("count,length,group,window", CASES)
def test_the_bound(count, length, group, window, size, asym):
    gen = torch.Generator().manual_seed(count + length)
    k, km = cached(length, asym, gen)
    v, vm = cached(length, asym, gen)
    # queries whose softmax is broad, so that every token counts (a narrow one's tokens are mostly nothing, and so is what losing them does)
    x = size * torch.randn((count, 2, group, 128), generator=gen, dtype=torch.float64)
    few, scale = count * group <= 16, 128 ** -0.5
    seen = kv_norms.seen_by(length, count, True, window, "cpu")
    o, bound = kv_norms.attend(x, k, km, v, vm, seen, scale, few)
    inside = lambda y: (y - o).norm(dim=-1) <= bound  # noqa: E731
    assert bool(inside(kernel_like(x, k, km, v, vm, seen, scale, few)).all())
    share = lambda y: float(inside(y).double().mean())  # noqa: E731
    assert share(torch.zeros_like(o)) == 0
    # rows off by 5 %: in any direction, and in size
    off = torch.randn(o.shape, generator=gen, dtype=torch.float64)
    assert share(o + 0.05 * off / off.norm(dim=-1, keepdim=True) * o.norm(dim=-1, keepdim=True)) == 0 and share(1.05 * o) == 0

    if size > 1:
        return

    def found(mask):
        """The share of the rows that see other tokens by this mask and are found out."""
        moved = (mask != seen).any(-1) & mask.any(-1)
        return float((~inside(kv_norms.attend(x, k, km, v, vm, mask, scale, few)[0]))[moved].double().mean())
    # a unit of 32 tokens is lost
    t, at = torch.arange(length), max(0, length - count - (16 if window else 64))
    assert found(seen & ((t < at) | (t >= at + 32))[None]) >= 0.95
    # the newest token is not seen, or the oldest; or one more than causality or the window allows is
    newest = t[None] == (length - count + torch.arange(count))[:, None]
    if length <= 1000:
        assert found(seen & ~newest) >= 0.95 and found(seen & (t > 0)[None]) >= 0.95 or window
        assert found(kv_norms.seen_by(length, count, True, window + 1, "cpu")) >= 0.95 or not window
        assert found(seen | (t[None] == (length - count + 1 + torch.arange(count))[:, None])) >= 0.95 or count == 1


# ----------------------------------------------------------------------------------------------
# the kernels
# ----------------------------------------------------------------------------------------------
HEADS = [(32, 8, 128), (8, 8, 80), (16, 1, 128), (14, 2, 64), (5, 5, 8), (40, 2, 96), (1, 1, 128)]


def check(plan, lengths, counts, heads, kv_heads, page, seed=0, order=None, max_len=0, **kw):
    """With a softmax that is broad, where every token counts, and with a narrow one."""
    order = order or list(range(len(lengths)))
    cache = kv_util.filled(plan, lengths, kv_heads, page, seed=seed)
    gen = torch.Generator(device=kv_util.DEV)
    gen.manual_seed(seed + 1)
    d = plan.info.d
    counts = [counts[i] for i in order]
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=kv_util.DEV)  # noqa: E731
    for size in (0.5, 3.0):
        q = (torch.randn((sum(counts), heads, d), generator=gen, device=kv_util.DEV) * size * (128 / d) ** 0.5).to(torch.bfloat16)
        got = cache.attention(q, ints(order), ints(np.concatenate([[0], np.cumsum(counts)]).tolist()), max(counts), max_len=max_len, **kw)
        kv_norms.check(cache, got, q, order, counts, **kw)


def plan_of(d, asym):
    from paper_2504_13989_b200 import Plan
    from paper_2504_13989_b200 import build as gbs_build
    gbs_build.build()
    return Plan(d, 128, 1, 4, 128, 0.9, asymmetric=asym)


@pytest.mark.gpu
@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("heads,kv_heads,d", HEADS)
def test_single_tokens(heads, kv_heads, d, asym):
    with plan_of(d, asym) as plan:
        for page in (16, 32, 64, 128):
            check(plan, [1, 15, 16, 17, 63, 129, 0, 300, 1000], [1] * 9, heads, kv_heads, page, seed=page, order=[8, 1, 0, 2, 6, 3, 4, 5, 7])
            check(plan, [1000, 20, 700, 4000], [1] * 4, heads, kv_heads, page, seed=page, window=20, scale=0.05)


@pytest.mark.gpu
@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("heads,kv_heads,d", HEADS)
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 33), (False, 33)])
def test_few_tokens(heads, kv_heads, d, causal, window, asym):
    with plan_of(d, asym) as plan:
        check(plan, [3, 40, 200, 2, 0, 513, 1], [3, 2, 4, 4, 1, 0, 1], heads, kv_heads, 32, causal=causal, window=window)


@pytest.mark.gpu
@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("heads,kv_heads,d,page", [(32, 8, 128, 16), (8, 8, 80, 64), (14, 2, 64, 128), (4, 1, 128, 32)])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 100), (False, 100)])
def test_prompts(heads, kv_heads, d, page, causal, window, asym):
    with plan_of(d, asym) as plan:
        check(plan, [130, 1, 700, 0, 64, 333, 20], [130, 1, 129, 2, 17, 333, 31], heads, kv_heads, page, order=[4, 0, 2, 1, 3, 5, 6], causal=causal, window=window)


@pytest.mark.gpu
@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("counts", [[1], [1, 1, 1], [2, 4], [100], [300, 40]])
def test_long_cache(counts, asym):
    with plan_of(128, asym) as plan:
        lengths = [40000, 300, 20011][:len(counts)]
        for window in (0, 9000):
            check(plan, lengths, counts, 8, 2, 64, window=window)


@pytest.mark.gpu
@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("counts", [[1, 1], [40, 2]])
def test_long_segments_in_one_block(counts, asym):
    """As in a large batch of long sequences, where a block goes through thousands of units of one: a small max_len has every segment undivided."""
    with plan_of(128, asym) as plan:
        check(plan, [60000, 130000], counts, 8, 2, 64, max_len=512)


@pytest.mark.gpu
@pytest.mark.parametrize("asym", [False, True])
def test_windows_at_every_offset(asym):
    with plan_of(64, asym) as plan:
        for counts in ([2], [130]):
            check(plan, [260], counts, 3, 1, 16, scale=-0.2)
            for window in (1, 2, 31, 32, 33, 64, 127, 128, 129):
                check(plan, [260], counts, 3, 1, 16, window=window)


@pytest.mark.gpu
def test_prompts_of_every_length_around_a_tile():
    with plan_of(128, False) as plan:
        for count in (6, 42, 43, 44, 85, 86, 87, 128, 171, 172):
            check(plan, [count, count + 1, count + 200], [count] * 3, 3, 1, 64, seed=count)
