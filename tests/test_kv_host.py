"""Refusals of the paged KV cache's calls, which need no device: every one is caught on the host, before anything is launched."""
import ctypes

import pytest

from paper_2504_13989_b200 import binding
from paper_2504_13989_b200 import build as gbs_build

OK, INVALID, UNSUPPORTED, ALIGN = binding.GBS_OK, binding.GBS_ERR_INVALID_ARG, binding.GBS_ERR_UNSUPPORTED, binding.GBS_ERR_ALIGNMENT
FIELDS = ("d", "d_pad", "m", "k", "bits", "group")


@pytest.fixture(scope="module")
def lib():
    gbs_build.build()
    return binding.lib()


def plan(d=128, d_pad=128, m=1, k=7, bits=4, group=128):
    """The start of a plan as the library keeps it (a plan needs a device): its sizes, and zeros behind them (symmetric, device 0)."""
    buf = ctypes.create_string_buffer(32768)
    ints = (ctypes.c_int * len(FIELDS)).from_buffer(buf)
    ints[:] = [d, d_pad, m, k, bits, group]
    return buf


def pool(**kw):
    f = dict(pages=1 << 20, n_pages=10, n_kv_heads=4, page_size=16, page_table=1 << 21, lengths=1 << 22, refs=1 << 23, n_seqs=5, max_pages=7)
    f.update(kw)
    return binding.KVCacheStruct(*f.values())


BAD_POOLS = [
    (dict(pages=None), INVALID), (dict(page_table=None), INVALID), (dict(lengths=None), INVALID), (dict(refs=None), INVALID),
    (dict(n_pages=0), INVALID), (dict(n_pages=(1 << 30) + 1), INVALID), (dict(n_kv_heads=0), INVALID), (dict(n_kv_heads=1025), INVALID),
    (dict(page_size=8), INVALID), (dict(page_size=48), INVALID), (dict(page_size=256), INVALID), (dict(n_seqs=0), INVALID),
    (dict(max_pages=0), INVALID), (dict(page_size=128, max_pages=1 << 24), INVALID),
    (dict(pages=(1 << 20) + 8), ALIGN), (dict(page_table=(1 << 21) + 2), ALIGN), (dict(lengths=(1 << 22) + 1), ALIGN), (dict(refs=(1 << 23) + 2), ALIGN),
]
P = 1 << 24                                                    # an address that no call here follows


def calls(lib, pl, c):
    """Every call on a pool with arguments that are right, for no items."""
    r = ctypes.byref(c)
    return {
        "extend": lib.gbs_kv_extend(pl, r, P, P, 0, P, None),
        "fork": lib.gbs_kv_fork(pl, r, P, P, 0, P, None),
        "free": lib.gbs_kv_free(pl, r, P, 0, None),
        "append": lib.gbs_kv_append(pl, r, P, P, 0, 0, P, P, 512, 128, None),
        "read": lib.gbs_kv_read(pl, r, P, P, 0, 0, P, P, None),
        "attention": lib.gbs_kv_attention(pl, r, P, P, 0, 0, 1, 0, P, 1024, 128, 8, 0.0, 0, 1, P, 1024, 128, P, 1 << 30, None),
    }


def test_calls_without_items_do_nothing(lib):
    assert set(calls(lib, plan(), pool()).values()) == {OK}


@pytest.mark.parametrize("change,want", BAD_POOLS)
def test_pools(lib, change, want):
    assert set(calls(lib, plan(), pool(**change)).values()) == {want}
    assert lib.gbs_kv_compact(plan(), ctypes.byref(pool(**change)), ctypes.byref(pool()), P, P, None) == want
    assert lib.gbs_kv_compact(plan(), ctypes.byref(pool()), ctypes.byref(pool(**change)), P, P, None) == want


@pytest.mark.parametrize("change", [dict(bits=3), dict(d=64, d_pad=64, k=6), dict(d_pad=256, k=8), dict(group=64), dict(group=32), dict(d=100)])
def test_plans(lib, change):
    pl = plan(**change)
    assert set(calls(lib, pl, pool()).values()) == {UNSUPPORTED}
    out = ctypes.c_int64(0)
    assert lib.gbs_kv_page_bytes(pl, 4, 16, ctypes.byref(out)) == UNSUPPORTED
    assert set(calls(lib, None, pool()).values()) == {INVALID}


def test_page_bytes(lib):
    out = ctypes.c_int64(0)
    for page in (16, 32, 64, 128):
        for heads in (1, 8, 1024):
            assert lib.gbs_kv_page_bytes(plan(), heads, page, ctypes.byref(out)) == OK and out.value == heads * page * 136
    for heads, page in ((0, 16), (1025, 16), (1, 8), (1, 20), (1, 256)):
        assert lib.gbs_kv_page_bytes(plan(), heads, page, ctypes.byref(out)) == INVALID
    assert lib.gbs_kv_page_bytes(plan(), 1, 16, None) == INVALID


def test_bookkeeping(lib):
    pl, c = plan(), pool()
    r = ctypes.byref(c)
    most = binding.GBS_KV_MAX_ITEMS
    for n in (-1, most + 1):
        assert lib.gbs_kv_extend(pl, r, P, P, n, P, None) == INVALID
        assert lib.gbs_kv_fork(pl, r, P, P, n, P, None) == INVALID
        assert lib.gbs_kv_free(pl, r, P, n, None) == INVALID
    assert lib.gbs_kv_extend(pl, r, None, None, 6, P, None) == INVALID              # more items than sequences
    assert lib.gbs_kv_free(pl, r, None, 6, None) == INVALID
    assert lib.gbs_kv_extend(pl, r, P, P, 1, None, None) == INVALID
    assert lib.gbs_kv_extend(pl, r, P + 2, P, 1, P, None) == ALIGN
    assert lib.gbs_kv_extend(pl, r, P, P + 1, 1, P, None) == ALIGN
    assert lib.gbs_kv_extend(pl, r, P, P, 1, P + 2, None) == ALIGN
    for a in ((None, P, P), (P, None, P), (P, P, None)):
        assert lib.gbs_kv_fork(pl, r, a[0], a[1], 1, a[2], None) == INVALID
    for a in ((P + 2, P, P), (P, P + 2, P), (P, P, P + 2)):
        assert lib.gbs_kv_fork(pl, r, a[0], a[1], 1, a[2], None) == ALIGN
    assert lib.gbs_kv_free(pl, r, P + 1, 1, None) == ALIGN


def test_compact(lib):
    pl, c = plan(), pool()
    other = dict(pages=3 << 20, page_table=5 << 21, lengths=5 << 22, refs=5 << 23)
    f = lambda into, m=P, n=P: lib.gbs_kv_compact(pl, ctypes.byref(c), ctypes.byref(into), m, n, None)  # noqa: E731
    for k in other:                                                                # an array that both pools have
        assert f(pool(**{a: v for a, v in other.items() if a != k})) == INVALID
    for k, v in (("n_kv_heads", 2), ("page_size", 32), ("n_seqs", 4), ("max_pages", 6)):
        assert f(pool(**other, **{k: v})) == INVALID
    into = pool(**other)
    assert f(into, None) == INVALID and f(into, P, None) == INVALID
    assert f(into, P + 2) == ALIGN and f(into, P, P + 1) == ALIGN
    assert lib.gbs_kv_compact(pl, None, ctypes.byref(into), P, P, None) == INVALID


def test_rows(lib):
    pl, c = plan(d=80), pool()
    r = ctypes.byref(c)
    a = lambda seqs=P, cu=P, n=2, t=3, k=P, v=P, ts=320, hs=80: lib.gbs_kv_append(pl, r, seqs, cu, n, t, k, v, ts, hs, None)  # noqa: E731
    assert a(n=-1) == INVALID and a(t=-1) == INVALID and a(cu=None) == INVALID     # three rows for two items of one token
    assert a(k=None) == INVALID and a(v=None) == INVALID and a(ts=72) == INVALID and a(hs=72) == INVALID
    assert a(ts=324) == ALIGN and a(hs=84) == ALIGN and a(k=P + 8) == ALIGN and a(v=P + 2) == ALIGN and a(cu=P + 2) == ALIGN and a(seqs=P + 1) == ALIGN
    assert a(t=1 << 28) == INVALID and a(t=1 << 62) == INVALID                      # rows x heads
    assert a(seqs=None, n=6) == INVALID
    assert a(t=0, k=None) == OK and a(n=0, k=None) == OK
    b = lambda seqs=P, cu=P, n=2, t=3, k=P, v=P: lib.gbs_kv_read(pl, r, seqs, cu, n, t, k, v, None)  # noqa: E731
    assert b(n=-1) == INVALID and b(t=-1) == INVALID and b(cu=None) == INVALID and b(k=None) == INVALID and b(v=None) == INVALID
    assert b(k=P + 8) == ALIGN and b(v=P + 2) == ALIGN and b(t=0, k=None) == OK


def test_attention(lib):
    pl, c = plan(d=80), pool()
    r = ctypes.byref(c)

    def f(seqs=P, cu=P, n=2, t=3, most=2, long=0, q=P, qt=640, qh=80, heads=8, scale=0.0, window=0, flags=1, out=P, ot=640, oh=80, work=P, size=1 << 40):
        return lib.gbs_kv_attention(pl, r, seqs, cu, n, t, most, long, q, qt, qh, heads, scale, window, flags, out, ot, oh, work, size, None)
    assert f(heads=6) == INVALID and f(heads=0) == INVALID and f(heads=4 * 1025) == INVALID and f(most=0) == INVALID
    assert f(cu=None, n=3, most=2) == INVALID and f(cu=None) == INVALID and f(most=1 << 30) == INVALID
    assert f(scale=float("inf")) == INVALID and f(scale=float("nan")) == INVALID and f(window=-1) == INVALID and f(flags=2) == INVALID and f(long=-1) == INVALID
    assert f(q=None) == INVALID and f(out=None) == INVALID and f(work=None) == INVALID and f(size=0) == INVALID
    assert f(qt=72) == INVALID and f(oh=72) == INVALID and f(qt=641) == ALIGN and f(oh=84) == ALIGN
    assert f(q=P + 8) == ALIGN and f(out=P + 4) == ALIGN and f(work=P + 8) == ALIGN and f(seqs=P + 1) == ALIGN
    assert f(t=0, q=None) == OK and f(n=0, q=None) == OK
    size = ctypes.c_int64(-1)
    assert lib.gbs_kv_attention_workspace(pl, r, 8, 3, 2, ctypes.byref(size)) == OK and size.value > 0
    assert f(size=size.value - 1) == INVALID
    assert lib.gbs_kv_attention_workspace(pl, r, 8, 3, 2, None) == INVALID
    assert lib.gbs_kv_attention_workspace(pl, r, 6, 3, 2, ctypes.byref(size)) == INVALID
    assert lib.gbs_kv_attention_workspace(pl, r, 8, -1, 2, ctypes.byref(size)) == INVALID


def test_the_widest_table_and_one_beyond(lib):
    assert set(calls(lib, plan(), pool(max_pages=1 << 20, page_size=128)).values()) == {OK}
    assert set(calls(lib, plan(), pool(max_pages=(1 << 20) + 1)).values()) == {INVALID}


def test_attention_in_place_is_refused(lib):
    c = pool()
    f = lambda q, out: lib.gbs_kv_attention(plan(), ctypes.byref(c), P, P, 2, 3, 2, 0, q, 1024, 128, 8, 0.0, 0, 1, out, 1024, 128, P, 1 << 40, None)  # noqa: E731
    assert f(P, P) == INVALID


def test_numbers_beyond_32_bits_are_not_cut(lib):
    for heads, page in ((2 ** 32 + 2, 16), (2, 2 ** 32 + 16)):
        with pytest.raises(ValueError):
            binding.gbs_kv_page_bytes(ctypes.addressof(plan()), heads, page)
