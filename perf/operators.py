"""Performance cases of the paged KV cache held in four bits: what a serving loop does with it in a step.

  write     the step's new keys and values are rotated, quantized and written into their pages, and read back as bf16 rows
  attend    attention over the cache: single tokens, few tokens, chunks of prompts and whole prompts
  pages     the bookkeeping of a step: sequences end, new ones get pages, others are forked (shared pages, a copied last one)
  compact   the pages in use move into a smaller pool, in order

A cache is a pool of pages.  Page p holds, for each KV head, `page` tokens: their key codes (64 bytes a token, two per byte, the even
coordinate in the low half), their value codes, their key scales and their value scales (one fp32 Delta a token, or a (Delta, lo) pair).
Codes are those of the rotated row H x / sqrt(128), x padded to 128 coordinates.  table[s] lists the pages of sequence s, lengths[s] its tokens,
refs[p] how many sequences hold page p.
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEV = "cuda:0"
D = 128                                                          # coordinates of a rotated row


# ----------------------------------------------------------------------------------------------
# cases
# ----------------------------------------------------------------------------------------------
def _write(name, seqs, tokens, kv_heads, d=128, page=64, asym=False, mix=0):
    return {"name": name, "kind": "write", "seqs": seqs, "tokens": tokens, "kv_heads": kv_heads, "d": d, "page": page, "asym": asym, "mix": mix}


def _attend(name, seqs, kv, q, heads, kv_heads, d=128, page=64, asym=False, ragged=False, window=0, mix=0):
    return {"name": name, "kind": "attend", "seqs": seqs, "kv": kv, "q": q, "heads": heads, "kv_heads": kv_heads, "d": d, "page": page, "asym": asym,
            "ragged": ragged, "window": window, "mix": mix}


def _pages(name, seqs, kv, kv_heads, page=16, mix=0):
    return {"name": name, "kind": "pages", "seqs": seqs, "kv": kv, "kv_heads": kv_heads, "page": page, "mix": mix}


def _compact(name, pages, seqs, kv_heads, page=64, asym=False, mix=0):
    return {"name": name, "kind": "compact", "pages": pages, "seqs": seqs, "kv_heads": kv_heads, "page": page, "asym": asym, "mix": mix}


def listed():
    return [
        # one decoding step of 48 sequences: a token each
        _write("write_step", 48, 1, 8),
        # the prompts of seven requests, 2000 tokens each on average, written at once; the quantizer the paper takes for the cache
        _write("write_prompts", 7, 2000, 8, asym=True, mix=1),
        # one user's chat: a single token against a short context, where the call's own latency counts
        _attend("attend_one", 1, 300, 1, 32, 8, page=16),
        # a busy decoding step: 64 sequences from a few tokens to 4096, small pages
        _attend("attend_step", 64, 4096, 1, 32, 8, page=16, ragged=True, mix=2),
        # 16 sequences x 32 heads x 4096 tokens, as many KV heads as query heads, asymmetric
        _attend("attend_mha", 16, 4096, 1, 32, 32, asym=True, mix=3),
        # two long documents, few rows: the long axis has to be split
        _attend("attend_long", 2, 131000, 1, 64, 8, page=128, mix=4),
        # a chunk of 2048 prompt tokens behind 6000 cached ones
        _attend("attend_chunk", 1, 8048, 2048, 32, 8, mix=5),
        # whole prompts of several requests at once, heads of 80 coordinates expanded to 128
        _attend("attend_prompts", 6, 1700, 1700, 16, 4, d=80, ragged=True, mix=6),
        # a beam search step of 24 sequences
        _pages("pages_few", 24, 700, 8, mix=7),
        # a large server's step: 1024 sequences of up to 2000 tokens, of which a quarter is forked anew and an eighth replaced
        _pages("pages_many", 1024, 2000, 8, mix=8),
        # a small pool that shrinks
        _compact("compact_few", 150, 20, 8, mix=9),
        # a pool of half a gigabyte that shrinks
        _compact("compact_many", 8192, 300, 8, mix=10),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm; odd ones among them."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["write", "attend", "attend", "attend", "prompt", "prompt", "pages", "compact"])
    mix, page, asym = rng.randrange(1 << 20), rng.choice([16, 32, 64, 128]), rng.random() < 0.4
    d = rng.choice([128, 128, 128, 64, 80, 96, 112])
    if kind == "write":
        seqs, kv_heads = _log(rng, 1, 64), rng.choice([1, 2, 4, 8, 32])
        c = _write("", seqs, _log(rng, 1, max(1, 112000 // (seqs * kv_heads))), kv_heads, d, page, asym, mix)
    elif kind == "attend":
        kv_heads, group = rng.choice([(1, 8), (2, 4), (4, 4), (8, 1), (8, 4), (8, 8), (32, 1)])
        seqs = _log(rng, 1, 128)
        q = rng.choice([1, 1, 1, 2, 4])
        kv = max(q, _log(rng, 1, max(1, min(131000, 2000000 // (seqs * kv_heads)))))
        c = _attend("", seqs, kv, q, kv_heads * group, kv_heads, d, page, asym, rng.random() < 0.5, rng.choice([0, 0, 0, 1024]), mix)
    elif kind == "prompt":
        kv_heads, group = rng.choice([(2, 4), (4, 4), (8, 1), (8, 4), (4, 7)])
        seqs, q = _log(rng, 1, 6), _log(rng, 17, 1500)
        kv = q + rng.choice([0, 0, _log(rng, 1, 4000)])
        if seqs * q * kv * kv_heads * group > 400000000:
            seqs, q, kv = 1, min(q, 600), min(kv, 600 + kv - q)
        c = _attend("", seqs, kv, q, kv_heads * group, kv_heads, d, page, asym, rng.random() < 0.5, rng.choice([0, 0, 0, 512]), mix)
    elif kind == "pages":
        c = _pages("", _log(rng, 8, 1024), _log(rng, 20, 2000), rng.choice([1, 2, 4, 8]), rng.choice([16, 32]), mix)
    else:
        kv_heads = rng.choice([1, 2, 4, 8])
        c = _compact("", _log(rng, 20, 8192 * 16 // page // kv_heads * 2), _log(rng, 2, 300), kv_heads, page, asym, mix)
    del c["name"]
    return c


def _mixed(case, n, top):
    """n lengths of a ragged batch, 1 .. top, spread over their logarithm with one at the top."""
    rng = random.Random(case["mix"] * 7919 + n)
    v = [_log(rng, max(1, top // 64), top) for _ in range(n)]
    v[rng.randrange(n)] = top
    return v


def _lengths(case):
    """(tokens of the cache, new tokens) of each sequence."""
    n = case["seqs"]
    if case["kind"] == "write":
        new = _mixed(case, n, 2 * case["tokens"]) if case["tokens"] > 1 else [1] * n
        if case["tokens"] > 1:
            new = [max(1, v * n * case["tokens"] // sum(new)) for v in new]
        rng = random.Random(case["mix"])
        return [v + (rng.randrange(200) if case["tokens"] == 1 else 0) for v in new], new
    if case["ragged"]:
        kv = _mixed(case, n, case["kv"])
        return kv, [max(1, min(v, v * case["q"] // case["kv"])) for v in kv]
    return [case["kv"]] * n, [case["q"]] * n


# ----------------------------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------------------------
_plans = {}


def _plan(d, asym):
    """The plan that a program keeps for its cache."""
    from paper_2504_13989_b200 import Plan
    if (d, asym) not in _plans:
        _plans[d, asym] = Plan(d, D, 1, 4, 128, 1.0 if asym else 0.9, asymmetric=asym)
    return _plans[d, asym]


def _fill(pages, n_pages, kv_heads, page, asym, gen):
    """Codes and scales as the quantizer leaves them for rows whose size varies from token to token; a few pages at a time."""
    sf = 2 if asym else 1
    blocks = pages.view(n_pages, kv_heads, -1)
    floats = pages.view(torch.float32).view(n_pages, kv_heads, -1)
    step = max(1, (1 << 28) // (kv_heads * page * 256))
    for a in range(0, n_pages, step):
        n = min(step, n_pages - a)
        y = torch.randn((n, kv_heads, page * 256), generator=gen, device=DEV, dtype=torch.float16).mul_(2.6)
        y = (y.add_(7.5).round_().clamp_(0, 15) if asym else y.round_().clamp_(-7, 7)).to(torch.int8)
        y = (y & 15).view(n, kv_heads, -1, 2)
        blocks[a:a + n, :, :page * 128] = (y[..., 0] | (y[..., 1] << 4)).view(torch.uint8)
        size = torch.randn((n, kv_heads, 2 * page, sf), generator=gen, device=DEV).mul_(0.25).exp_().mul_(0.3)
        if asym:
            size[..., 1] = size[..., 0] * (-7.5 + 0.5 * torch.randn((n, kv_heads, 2 * page), generator=gen, device=DEV))
        floats[a:a + n, :, page * 32:] = size.view(n, kv_heads, -1)


def _new_cache(lengths, kv_heads, page, asym, gen, spare=8, n_pages=None, seqs=None, filled=True):
    """A pool in use: the pages of the sequences lie in no order, some are free."""
    need = [-(-v // page) for v in lengths]
    n_pages = sum(need) + spare if n_pages is None else n_pages
    block = page * (128 + 8 * (2 if asym else 1))
    pages = torch.zeros((n_pages, kv_heads * block), dtype=torch.uint8, device=DEV)
    if filled:
        _fill(pages, n_pages, kv_heads, page, asym, gen)
    order = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
    seqs = len(lengths) if seqs is None else seqs
    table = torch.full((seqs, max(need) + 2), -1, dtype=torch.int32, device=DEV)
    held = torch.tensor(need, device=DEV)
    at = torch.repeat_interleave(torch.arange(len(need), device=DEV), held)
    col = torch.arange(len(at), device=DEV) - (held.cumsum(0) - held)[at]
    table[at, col] = order[:len(at)]
    refs = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    refs[order[:len(at)].long()] = 1
    return {"pages": pages, "table": table, "lengths": torch.tensor(lengths + [0] * (seqs - len(lengths)), dtype=torch.int32, device=DEV), "refs": refs}


def _handle(plan, c, case):
    from paper_2504_13989_b200 import KVCache
    return KVCache(plan, c["pages"], c["table"], c["lengths"], c["refs"], case["kv_heads"], case["page"])


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = dict(case)
    kind = case["kind"]
    asym = case.get("asym", False)
    if kind in ("write", "attend"):
        kv, new = _lengths(case)
        n, d = case["seqs"], case["d"]
        s["cache"] = _new_cache(kv, case["kv_heads"], case["page"], asym, gen, filled=kind == "attend")
        # the items of a call are sequences in another order than the table's
        s["rows"] = torch.randperm(n, generator=torch.Generator().manual_seed(case["mix"])).to(DEV, torch.int32)
        new = [new[i] for i in s["rows"].tolist()]
        s["max_new"], s["total"], s["longest"] = max(new), sum(new), max(kv)
        s["cu"] = torch.tensor([0] + new, dtype=torch.int32, device=DEV).cumsum(0).to(torch.int32)
        if kind == "write":
            k = torch.randn((s["total"], case["kv_heads"], d), generator=gen, device=DEV)
            k[:, :, [3, d // 2 + 1]] *= 8.0                       # keys have a few large channels
            s["k"] = k.to(torch.bfloat16)
            s["v"] = torch.randn((s["total"], case["kv_heads"], d), generator=gen, device=DEV).to(torch.bfloat16)
        else:
            s["q"] = (torch.randn((s["total"], case["heads"], d), generator=gen, device=DEV) * 3.0 * math.sqrt(D / d)).to(torch.bfloat16)
    elif kind == "pages":
        n = case["seqs"]
        kv = _mixed(case, n, case["kv"])
        # every sequence can be replaced by the longest
        s["cache"] = _new_cache(kv, case["kv_heads"], case["page"], asym, gen, n_pages=sum(-(-v // case["page"]) for v in kv) + n * (case["kv"] // case["page"] + 1) // 2)
        order = torch.randperm(n, generator=torch.Generator().manual_seed(case["mix"])).to(DEV, torch.int32)
        forks, fresh = n // 4, n // 8
        s["dst"], s["fresh"], s["ended"] = order[:forks].contiguous(), order[forks:forks + fresh].contiguous(), order[:forks + fresh].contiguous()
        rest = order[forks + fresh:]
        s["src"] = rest[torch.randint(len(rest), (forks,), generator=gen, device=DEV)].contiguous()
        s["counts"] = torch.randint(1, case["kv"] + 1, (fresh,), generator=gen, device=DEV).to(torch.int32)
    else:
        live = max(1, case["pages"] * 6 // 10)
        n = min(case["seqs"], live)
        per = [live // n + (i < live % n) for i in range(n)]
        rng = random.Random(case["mix"])
        kv = [p * case["page"] - rng.randrange(case["page"]) for p in per]
        s["cache"] = _new_cache(kv, case["kv_heads"], case["page"], asym, gen, n_pages=case["pages"])
        c = s["cache"]
        s["into"] = {"pages": torch.zeros((live + live // 20 + 1, c["pages"].shape[1]), dtype=torch.uint8, device=DEV), "table": torch.zeros_like(c["table"]),
                     "lengths": torch.zeros_like(c["lengths"]), "refs": torch.zeros(live + live // 20 + 1, dtype=torch.int32, device=DEV)}
    if own:
        plan = _plan(case.get("d", D), asym)
        s["handle"] = _handle(plan, s["cache"], case)
        if kind == "compact":
            s["into_handle"] = _handle(plan, s["into"], case)
    return s


# ----------------------------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------------------------
def run(s):
    kind = s["kind"]
    c = s["cache"]
    if own:
        h = s["handle"]
        if kind == "write":
            h.append(s["k"], s["v"], s["rows"], s["cu"])
            return h.read(s["rows"], s["cu"], s["total"])
        if kind == "attend":
            return h.attention(s["q"], s["rows"], s["cu"], s["max_new"], window=s["window"], max_len=s["longest"])
        if kind == "pages":
            h.free(s["ended"])
            status = h.extend(s["fresh"], s["counts"]), h.fork(s["src"], s["dst"])
            return status, c["table"], c["lengths"], c["refs"], c["pages"].view(torch.int32)
        into = s["into"]
        live = h.compact(s["into_handle"])
        return live, into["table"], into["lengths"], into["refs"], into["pages"].view(torch.int32)
    if kind == "write":
        _plain_append(s)
        return _plain_read(s)
    if kind == "attend":
        return _plain_attention(s)
    if kind == "pages":
        _plain_free(c, s["ended"].long(), s["page"])
        status = _plain_extend(c, s["fresh"].long(), s["counts"], s["page"]), _plain_fork(c, s["src"].long(), s["dst"].long(), s["page"], s["kv_heads"])
        return status, c["table"], c["lengths"], c["refs"], c["pages"].view(torch.int32)
    live = _plain_compact(c, s["into"], s["page"])
    into = s["into"]
    return live, into["table"], into["lengths"], into["refs"], into["pages"].view(torch.int32)


# ----------------------------------------------------------------------------------------------
# the plain form
# ----------------------------------------------------------------------------------------------
_h = {}


def _hadamard(dtype):
    """H_128 by Sylvester's recursion, as signs."""
    if dtype not in _h:
        h2 = torch.tensor([[1, 1], [1, -1]], dtype=torch.float64)
        _h[dtype] = torch.kron(torch.kron(torch.kron(h2, h2), torch.kron(h2, h2)), torch.kron(h2, torch.kron(h2, h2))).to(DEV, dtype)
    return _h[dtype]


def _where(s):
    """(sequence, position) of each of the call's tokens: the last ones of their sequences."""
    rows, cu = s["rows"].long(), s["cu"].long()
    item = torch.searchsorted(cu[1:], torch.arange(s["total"], device=DEV), right=True)
    count = cu[1:] - cu[:-1]
    return rows[item], s["cache"]["lengths"].long()[rows[item]] - count[item] + torch.arange(s["total"], device=DEV) - cu[item]


def _views(s):
    """The codes and scales of the pool: [pages, heads, page, 64] bytes and [pages, heads, page, 1 or 2] floats, keys' and values'."""
    page, sf = s["page"], 2 if s["asym"] else 1
    b = s["cache"]["pages"].view(s["cache"]["pages"].shape[0], s["kv_heads"], -1)
    f = b.view(torch.float32)
    a = page * 32
    return (b[..., :page * 64].unflatten(-1, (page, 64)), b[..., page * 64:page * 128].unflatten(-1, (page, 64)),
            f[..., a:a + page * sf].unflatten(-1, (page, sf)), f[..., a + page * sf:a + 2 * page * sf].unflatten(-1, (page, sf)))


def _plain_quantize(x, asym):
    """Rows of d coordinates -> packed codes, scales; next to a rounding border 32 bits would not do."""
    y = torch.nn.functional.pad(x.double(), (0, D - x.shape[-1])) @ _hadamard(torch.float64) / math.sqrt(D)
    if asym:
        lo, hi = y.amin(-1, keepdim=True), y.amax(-1, keepdim=True)
        delta = (hi - lo) / 15
        q = torch.where(delta > 0, (y - lo) / delta, 0).round().clamp(0, 15)
        scales = torch.cat([delta, lo], -1)
    else:
        delta = 0.9 * y.abs().amax(-1, keepdim=True) / 7
        q = torch.where(delta > 0, y / delta, 0).round().clamp(-7, 7)
        scales = delta
    q = (q.to(torch.int8) & 15).unflatten(-1, (64, 2))
    return (q[..., 0] | (q[..., 1] << 4)).view(torch.uint8), scales.float()


def _plain_values(codes, scales, asym):
    """yhat of packed codes and scales, fp32."""
    q = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    if asym:
        return q.float() * scales[..., :1] + scales[..., 1:]
    return ((q ^ 8).to(torch.int8) - 8).float() * scales


def _plain_append(s):
    seq, pos = _where(s)
    page, slot = s["cache"]["table"][seq, pos // s["page"]].long(), pos % s["page"]
    kc, vc, ks, vs = _views(s)
    kc[page, :, slot], ks[page, :, slot] = _plain_quantize(s["k"], s["asym"])
    vc[page, :, slot], vs[page, :, slot] = _plain_quantize(s["v"], s["asym"])


def _plain_read(s):
    seq, pos = _where(s)
    page, slot = s["cache"]["table"][seq, pos // s["page"]].long(), pos % s["page"]
    kc, vc, ks, vs = _views(s)
    back = _hadamard(torch.float32)[:, :s["d"]] / math.sqrt(D)
    return ((_plain_values(kc[page, :, slot], ks[page, :, slot], s["asym"]) @ back).to(torch.bfloat16),
            (_plain_values(vc[page, :, slot], vs[page, :, slot], s["asym"]) @ back).to(torch.bfloat16))


def _plain_attention(s):
    c, page, d, heads, kvh = s["cache"], s["page"], s["d"], s["heads"], s["kv_heads"]
    rows, cu = s["rows"].long(), s["cu"].long()
    n, mq, length = len(rows), s["max_new"], c["lengths"].long()[rows]
    held = c["table"][rows, :-(-s["longest"] // page)].long().clamp(min=0)
    kc, vc, ks, vs = _views(s)
    k, v = (_plain_values(b[held], f[held], s["asym"]).transpose(1, 2).flatten(2, 3) for b, f in ((kc, ks), (vc, vs)))   # [n, kv heads, tokens, 128]
    j = torch.arange(mq, device=DEV)
    count = cu[1:] - cu[:-1]
    at = (cu[:-1, None] + j).clamp(max=s["total"] - 1)
    q = torch.nn.functional.pad(s["q"].float(), (0, D - d)) @ (_hadamard(torch.float32) / math.sqrt(D))
    q = q[at].view(n, mq, kvh, heads // kvh, D).permute(0, 2, 3, 1, 4).flatten(2, 3)                                     # [n, kv heads, group * mq, 128]
    score = (q @ k.transpose(-1, -2) / math.sqrt(d)).view(n, kvh, heads // kvh, mq, -1)
    pos = length[:, None] - count[:, None] + j
    t = torch.arange(score.shape[-1], device=DEV)
    seen = (t <= pos[..., None]) & (t < length[:, None, None]) & (j < count[:, None])[..., None]
    if s["window"]:
        seen &= t > pos[..., None] - s["window"]
    seen = seen[:, None, None]
    score = score.masked_fill(~seen, float("-inf"))
    top = score.amax(-1, keepdim=True)
    p = torch.where(seen, torch.exp(score - torch.where(top > float("-inf"), top, 0)), 0)
    total = p.sum(-1, keepdim=True)
    o = (p / torch.where(total > 0, total, 1)).flatten(2, 3) @ v @ (_hadamard(torch.float32)[:, :d] / math.sqrt(D))
    o = o.view(n, kvh, heads // kvh, mq, d).permute(0, 3, 1, 2, 4).reshape(n, mq, heads, d)
    return o[j < count[:, None]].to(torch.bfloat16)


def _held(c, seqs, page):
    """Which entries of these sequences' rows of the table hold pages."""
    return torch.arange(c["table"].shape[1], device=DEV) < ((c["lengths"][seqs] + page - 1) // page)[:, None]


def _plain_free(c, seqs, page):
    ids = c["table"][seqs][_held(c, seqs, page)].long()
    c["refs"].index_add_(0, ids, torch.full_like(ids, -1, dtype=torch.int32))
    c["lengths"][seqs] = 0


def _plain_extend(c, seqs, counts, page):
    before = c["lengths"][seqs]
    first = (before + page - 1) // page
    need = ((before + counts + page - 1) // page - first).long()
    ids = torch.nonzero(c["refs"] == 0)[:, 0][:int(need.sum())]
    at = torch.repeat_interleave(torch.arange(len(seqs), device=DEV), need)
    c["table"][seqs[at], first[at] + torch.arange(len(at), device=DEV) - (need.cumsum(0) - need)[at]] = ids.to(torch.int32)
    c["refs"][ids] = 1
    c["lengths"][seqs] = before + counts
    return torch.zeros(len(seqs), dtype=torch.int32, device=DEV)


def _plain_fork(c, src, dst, page, kv_heads):
    length = c["lengths"][src]
    full, tail = length // page, length % page
    shared = torch.arange(c["table"].shape[1], device=DEV) < full[:, None]
    c["table"][dst] = torch.where(shared, c["table"][src], c["table"][dst])
    ids = c["table"][src][shared].long()
    c["refs"].index_add_(0, ids, torch.ones_like(ids, dtype=torch.int32))
    cut = tail > 0
    a, b, full, tail = src[cut], dst[cut], full[cut].long(), tail[cut]
    ids = torch.nonzero(c["refs"] == 0)[:, 0][:len(a)]
    c["refs"][ids] = 1
    c["table"][b, full] = ids.to(torch.int32)
    c["lengths"][dst] = length
    pool = c["pages"].view(c["pages"].shape[0], kv_heads, -1)
    byte = torch.arange(pool.shape[2], device=DEV)
    sized = (pool.shape[2] - page * 128) // (2 * page)
    token = torch.where(byte < page * 128, byte // 64, (byte - page * 128) // sized) % page
    pool[ids] = torch.where((token < tail[:, None])[:, None], pool[c["table"][a, full].long()], pool[ids])
    return torch.zeros(len(src), dtype=torch.int32, device=DEV)


def _plain_compact(c, into, page):
    used = c["refs"] > 0
    new = torch.where(used, used.cumsum(0) - 1, -1).to(torch.int32)
    ids = torch.nonzero(used)[:, 0]
    into["pages"][:len(ids)] = c["pages"][ids]
    into["refs"].zero_()
    into["refs"][:len(ids)] = c["refs"][ids]
    held = torch.arange(c["table"].shape[1], device=DEV) < ((c["lengths"] + page - 1) // page)[:, None]
    into["table"].copy_(torch.where(held, new[c["table"].long().clamp(min=0)], -1))
    into["lengths"].copy_(c["lengths"])
    return used.sum().to(torch.int32).reshape(1)


# ----------------------------------------------------------------------------------------------
# the definition in 64 bits, one sequence at a time and in the rows' own basis
# ----------------------------------------------------------------------------------------------
def _signs():
    i = torch.arange(D, device=DEV)
    x = i[:, None] & i[None, :]
    parity = sum((x >> b) & 1 for b in range(7)) % 2
    return 1.0 - 2.0 * parity.double()


def _exact_rows(s, seq, count):
    """The first `count` cached tokens of a sequence as rows of their own basis: [kv heads, count, d] keys and values."""
    c, page, sf = s["cache"], s["page"], 2 if s["asym"] else 1
    ids = c["table"][seq, :-(-count // page)].long()
    blocks = c["pages"][ids].view(len(ids), s["kv_heads"], -1)
    out = []
    for i in range(2):
        codes = blocks[:, :, i * page * 64:(i + 1) * page * 64].reshape(len(ids), s["kv_heads"], page, 64)
        at = page * 128 + i * page * 4 * sf
        scales = blocks[:, :, at:at + page * 4 * sf].contiguous().view(torch.float32).reshape(len(ids), s["kv_heads"], page, sf).double()
        y = torch.empty(codes.shape[:3] + (D,), dtype=torch.float64, device=DEV)
        y[..., 0::2], y[..., 1::2] = (codes % 16).double(), (codes // 16).double()
        y = y * scales[..., :1] + scales[..., 1:] if s["asym"] else (y - 16 * (y > 7)) * scales
        out.append((y.movedim(1, 0).flatten(1, 2)[:, :count] @ _signs() / D ** 0.5)[..., :s["d"]])
    return out


def exact(case, seed):
    if case["kind"] in ("pages", "compact"):
        return None                                              # whole numbers and bytes that move
    s = prepare(case, seed)
    if case["kind"] == "write":
        back = []
        for x in (s["k"], s["v"]):
            y = torch.zeros(x.shape[:2] + (D,), dtype=torch.float64, device=DEV)
            y[..., :s["d"]] = x
            y = y @ _signs() / D ** 0.5
            if s["asym"]:
                low = y.min(-1, keepdim=True).values
                step = (y.max(-1, keepdim=True).values - low) / 15
                y = torch.floor((y - low) / step + 0.5).clamp_(0, 15) * step + low
            else:
                step = y.abs().max(-1, keepdim=True).values * 0.9 / 7
                y = torch.round(y / step).clamp_(-7, 7) * step
            back.append((y @ _signs() / D ** 0.5)[..., :s["d"]])
        return tuple(back)
    group = case["heads"] // case["kv_heads"]
    cu, rows, lengths = s["cu"].tolist(), s["rows"].tolist(), s["cache"]["lengths"].tolist()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    for i, seq in enumerate(rows):
        count, length = cu[i + 1] - cu[i], lengths[seq]
        k, v = _exact_rows(s, seq, length)
        for a in range(0, count, 256):                           # some query tokens at a time
            b = min(count, a + 256)
            q = s["q"][cu[i] + a:cu[i] + b].double().view(b - a, case["kv_heads"], group, case["d"])
            score = torch.einsum("qhgd,hkd->qhgk", q, k) / case["d"] ** 0.5
            far = (length - count + torch.arange(a, b, device=DEV))[:, None] - torch.arange(length, device=DEV)
            hidden = (far < 0) | (far >= case["window"]) if case["window"] else far < 0
            p = torch.softmax(score.masked_fill(hidden[:, None, None], -math.inf), -1)
            out[cu[i] + a:cu[i] + b] = torch.einsum("qhgk,hkd->qhgd", p, v).reshape(b - a, case["heads"], case["d"])
    return out


# ----------------------------------------------------------------------------------------------
# what a pass cannot do without
# ----------------------------------------------------------------------------------------------
def work(case):
    kind, sf = case["kind"], 2 if case.get("asym") else 1
    token = 128 + 8 * sf                                         # bytes of a token and KV head in the cache
    if kind == "write":
        rows = sum(_lengths(case)[1]) * case["kv_heads"]
        return {"bytes": rows * (2 * 2 * case["d"] * 2 + token), "flops": rows * 4 * 128 * 7}
    if kind == "attend":
        kv, new = _lengths(case)
        window, pairs, read = case["window"], 0, 0
        for a, b in zip(kv, new):
            if window:
                pairs += sum(min(window, a - b + j + 1) for j in range(b))
                read += min(a, window + b - 1)
            else:
                pairs += b * (a - b) + b * (b + 1) // 2
                read += a
        return {"bytes": read * case["kv_heads"] * token + 2 * 2 * sum(new) * case["heads"] * case["d"], "flops": 4 * 128 * case["heads"] * pairs}
    if kind == "pages":
        n, page = case["seqs"], case["page"]
        kv = _mixed(case, n, case["kv"])
        mean = sum(-(-v // page) for v in kv) / n
        forks, fresh = n // 4, n // 8
        # entries of the table and counters of the pages that are let go, taken and shared, and half a page that each fork copies
        held = (forks + fresh) * mean + fresh * case["kv"] / 2 / page + forks * mean
        return {"bytes": held * 12 + forks * case["kv_heads"] * page * token, "flops": 0}
    live = max(1, case["pages"] * 6 // 10)
    return {"bytes": 2 * live * case["kv_heads"] * case["page"] * token, "flops": 0}
