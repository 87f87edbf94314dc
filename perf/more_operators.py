"""Performance cases of long contexts in the paged KV cache held in four bits: shared by many sequences, weighed, and cut down.

  shared    attention of sequences that share a prefix (forks of one prompt): the prefix is attended over once for all of a group
  mass      the softmax weight that each cached token got from a call's queries, added to what it had
  evict     sequences cut down to the tokens with the most weight, for each KV head its own, behind the first and before the last ones

A cache is a pool of pages.  Page p holds, for each KV head, `page` tokens: their key codes (64 bytes a token, two per byte, the even
coordinate in the low half), their value codes, their key scales and their value scales (one fp32 Delta a token, or a (Delta, lo) pair).
Codes are those of the rotated row H x / sqrt(128), x padded to 128 coordinates.  table[s] lists the pages of sequence s, lengths[s] its tokens,
refs[p] how many sequences hold page p.  Weights are kept beside it: mass[s][KV head][position].
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False
DEV = "cuda:0"
D = 128                                                          # coordinates of a rotated row


# ----------------------------------------------------------------------------------------------
# cases
# ----------------------------------------------------------------------------------------------
def _shared(name, seqs, groups, prefix, rest, q, heads, kv_heads, d=128, page=64, asym=False, mix=0):
    return {"name": name, "kind": "shared", "seqs": seqs, "groups": groups, "prefix": prefix, "rest": rest, "q": q, "heads": heads, "kv_heads": kv_heads,
            "d": d, "page": page, "asym": asym, "mix": mix}


def _mass(name, seqs, kv, q, heads, kv_heads, d=128, page=64, asym=False, ragged=False, window=0, decay=1.0, mix=0):
    return {"name": name, "kind": "mass", "seqs": seqs, "kv": kv, "q": q, "heads": heads, "kv_heads": kv_heads, "d": d, "page": page, "asym": asym,
            "ragged": ragged, "window": window, "decay": decay, "mix": mix}


def _evict(name, seqs, kv, keep, kv_heads, page=64, asym=False, mix=0):
    return {"name": name, "kind": "evict", "seqs": seqs, "kv": kv, "keep": keep, "kv_heads": kv_heads, "page": page, "asym": asym, "mix": mix}


def listed():
    return [
        # four answers sampled to one short question: the call's own latency counts
        _shared("shared_few", 4, 1, 300, 40, 1, 32, 8, page=16),
        # a busy decoding step behind one system prompt of 6000 tokens, 64 sequences with up to 300 tokens of their own
        _shared("shared_step", 64, 1, 6000, 300, 1, 32, 8, mix=1),
        # a decoding step of seven prompts with several samples each, short prompts and long ones, asymmetric, heads of 96 coordinates
        _shared("shared_groups", 40, 7, 8000, 500, 1, 28, 4, d=96, page=32, asym=True, mix=2),
        # twelve questions about one long document, four tokens each in a step (guessed ahead, to be verified)
        _shared("shared_long", 12, 1, 100000, 900, 4, 64, 8, page=128, mix=3),
        # the questions themselves: eight prompts of up to 250 tokens behind a document of 12000
        _shared("shared_prompts", 8, 1, 12000, 250, 250, 32, 8, mix=4),
        # one user's chat: the weights of a single token over a short context
        _mass("mass_one", 1, 300, 1, 32, 8, page=16, mix=5),
        # a decoding step of 48 sequences of up to 6000 tokens, asymmetric, what was there fades
        _mass("mass_step", 48, 6000, 1, 32, 8, asym=True, ragged=True, decay=0.98, mix=6),
        # the last 32 tokens of four prompts look back over what they will leave behind
        _mass("mass_window", 4, 9000, 32, 32, 8, ragged=True, decay=0.0, mix=7),
        # a chunk of 1000 prompt tokens behind 5000 cached ones, heads of 80 coordinates
        _mass("mass_chunk", 1, 6000, 1000, 16, 4, d=80, mix=8),
        # a few chats cut down to 256 tokens
        _evict("evict_few", 6, 700, 256, 8, page=16, mix=9),
        # a large server's step: 96 sequences of up to 4096 tokens, cut down to 1024, asymmetric
        _evict("evict_many", 96, 4096, 1024, 8, asym=True, mix=10),
        # two long documents, cut down to an eighth
        _evict("evict_long", 2, 131000, 16384, 8, page=128, mix=11),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm; odd ones among them."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["shared", "shared", "prompts", "mass", "mass", "evict"])
    mix, page, asym = rng.randrange(1 << 20), rng.choice([16, 32, 64, 128]), rng.random() < 0.4
    d = rng.choice([128, 128, 128, 64, 80, 96, 112])
    kv_heads, group = rng.choice([(1, 8), (2, 4), (4, 4), (4, 7), (8, 1), (8, 4), (8, 8)])
    if kind == "shared":
        seqs, q = _log(rng, 2, 96), rng.choice([1, 1, 1, 2, 4])
        groups = rng.choice([1, 1, _log(rng, 1, seqs)])
        prefix = _log(rng, 16, max(16, min(100000, 800000 // (groups * kv_heads), 500000000 // (seqs * q * kv_heads * group))))
        c = _shared("", seqs, groups, prefix, _log(rng, 8, 900), q, kv_heads * group, kv_heads, d, page, asym, mix)
    elif kind == "prompts":
        seqs = _log(rng, 2, 12)
        q = _log(rng, 17, 250)
        prefix = _log(rng, 100, max(100, min(12000, 500000000 // (seqs * q * kv_heads * group))))
        c = _shared("", seqs, rng.choice([1, 1, 2]), prefix, q + rng.choice([0, 0, 100]), q, kv_heads * group, kv_heads, d, page, asym, mix)
    elif kind == "mass":
        q = rng.choice([1, 1, 1, 4, 32, _log(rng, 1, 1000)])
        seqs = _log(rng, 1, 64 if q <= 4 else 4)
        kv = max(q, _log(rng, 8, max(8, min(100000, 2000000 // (seqs * kv_heads), 90000000 // (seqs * q * kv_heads * group)))))
        c = _mass("", seqs, kv, q, kv_heads * group, kv_heads, d, page, asym, rng.random() < 0.5, rng.choice([0, 0, 0, 512]), rng.choice([0.0, 0.98, 1.0]), mix)
    else:
        seqs = _log(rng, 1, 96)
        kv = _log(rng, 40, max(40, min(131000, 3000000 // (seqs * kv_heads))))
        c = _evict("", seqs, kv, max(2, kv // rng.choice([2, 3, 4, 8])), kv_heads, page, asym, mix)
    del c["name"]
    return c


def _mixed(case, n, top, least=1):
    """n lengths of a ragged batch, least .. top, spread over their logarithm with one at the top."""
    rng = random.Random(case["mix"] * 7919 + n)
    v = [_log(rng, max(least, top // 64), top) for _ in range(n)]
    v[rng.randrange(n)] = top
    return v


def _lengths(case):
    """(tokens of the cache, new tokens) of each sequence."""
    n = case["seqs"]
    if case["kind"] == "evict":
        return _mixed(case, n, case["kv"]), [0] * n
    if case["ragged"]:
        kv = _mixed(case, n, case["kv"])
        return kv, [max(1, min(v, case["q"])) for v in kv]
    return [case["kv"]] * n, [case["q"]] * n


def _family(case):
    """Of a shared case: (items of each group, tokens of each group's prefix, tokens of each item behind it, new tokens of each item)."""
    n, g = case["seqs"], case["groups"]
    rng = random.Random(case["mix"] * 104729 + n)
    cuts = sorted(rng.sample(range(1, n), g - 1)) if g > 1 else []
    sizes = [b - a for a, b in zip([0] + cuts, cuts + [n])]
    prefix = [case["prefix"]] if g == 1 else _mixed(case, g, case["prefix"])
    rest = [_log(rng, max(1, case["rest"] // 8), case["rest"]) for _ in range(n)]
    new = [max(1, min(case["q"], r)) for r in rest]
    return sizes, prefix, rest, new


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


def _new_cache(n_pages, held, lengths, seqs, width, case, gen):
    """A pool in use: `held` lists the pages of the first sequences by number, which lie in no order."""
    page, kv_heads, asym = case["page"], case["kv_heads"], case["asym"]
    pages = torch.zeros((n_pages, kv_heads * page * (128 + 8 * (2 if asym else 1))), dtype=torch.uint8, device=DEV)
    _fill(pages, n_pages, kv_heads, page, asym, gen)
    order = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
    table = torch.full((seqs, width), -1, dtype=torch.int32)
    for i, h in enumerate(held):
        table[i, :len(h)] = torch.tensor(h, dtype=torch.int32)
    table = table.to(DEV)
    table = torch.where(table >= 0, order[table.long().clamp(min=0)], -1)
    refs = torch.bincount(table[table >= 0].long(), minlength=n_pages).to(torch.int32)
    return {"pages": pages, "table": table, "lengths": torch.tensor(lengths + [0] * (seqs - len(lengths)), dtype=torch.int32, device=DEV), "refs": refs}


def _handle(plan, c, case):
    from paper_2504_13989_b200 import KVCache
    return KVCache(plan, c["pages"], c["table"], c["lengths"], c["refs"], case["kv_heads"], case["page"])


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = dict(case)
    kind, page, n = case["kind"], case["page"], case["seqs"]
    up = lambda v: -(-v // page)  # noqa: E731
    if kind == "shared":
        sizes, prefix, rest, new = _family(case)
        held, lengths, at = [], [], 0
        for size, p, first in zip(sizes, prefix, [sum(sizes[:i]) for i in range(len(sizes))]):
            common = list(range(at, at + p // page))             # forks share full pages
            at += len(common)
            for r in rest[first:first + size]:
                own_pages = up(p + r) - len(common)
                held.append(common + list(range(at, at + own_pages)))
                at += own_pages
                lengths.append(p + r)
        # a group's items stand together in a call, the sequences they are anywhere in the table
        place = torch.randperm(n, generator=torch.Generator().manual_seed(case["mix"]))
        back = torch.argsort(place).tolist()
        s["cache"] = _new_cache(at + 8, [held[i] for i in back], [lengths[i] for i in back], n, max(map(len, held)) + 2, case, gen)
        s["rows"] = place.to(DEV, torch.int32)
        s["cuts"] = torch.tensor([0] + sizes, dtype=torch.int32, device=DEV).cumsum(0).to(torch.int32)
        s["sizes"], s["prefix_tokens"], s["longest_rest"] = sizes, [p // page * page for p in prefix], max(rest) + page
    else:
        kv, new = _lengths(case)
        copies = n if kind == "evict" else 0                     # evict: sequences n .. 2 n - 1 are the short copies
        spare = sum(up(min(v, case["keep"])) + 1 for v in kv) if copies else 8
        ends = [sum(map(up, kv[:i + 1])) for i in range(n)]
        s["cache"] = _new_cache(ends[-1] + spare, [list(range(e - up(v), e)) for e, v in zip(ends, kv)], kv, n + copies, max(map(up, kv)) + 2, case, gen)
        s["rows"] = torch.randperm(n, generator=torch.Generator().manual_seed(case["mix"])).to(DEV, torch.int32)
        new = [new[i] for i in s["rows"].tolist()]
        s["longest"] = max(kv)
        # weights as they come about: few tokens have most of it, many have none at all
        w = torch.rand((n + copies, case["kv_heads"], max(kv)), generator=gen, device=DEV).pow_(6.0)
        s["base"] = torch.where(w < 1e-3, 0.0, w)
        s["mass"] = torch.zeros_like(s["base"])
    if kind == "evict":
        s["copies"] = s["rows"] + n
        s["base"][n:] = s["base"][:n].clone()
        s["first"], s["recent"] = min(4, case["keep"] // 4), case["keep"] // 4
    else:
        s["cu"] = torch.tensor([0] + new, dtype=torch.int32, device=DEV).cumsum(0).to(torch.int32)
        s["max_new"], s["total"] = max(new), sum(new)
        s["q"] = (torch.randn((s["total"], case["heads"], case["d"]), generator=gen, device=DEV) * 3.0 * math.sqrt(D / case["d"])).to(torch.bfloat16)
    if own:
        s["handle"] = _handle(_plan(case.get("d", D), case["asym"]), s["cache"], case)
    return s


# ----------------------------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------------------------
def run(s):
    kind, c = s["kind"], s["cache"]
    if kind == "shared":
        if own:
            return s["handle"].shared_attention(s["q"], s["rows"], s["cu"], s["cuts"], s["max_new"], max_own=s["longest_rest"])
        return _plain_shared(s)
    if kind == "mass":
        if own:
            return s["handle"].attention_mass(s["q"], s["mass"], s["rows"], s["cu"], s["max_new"], decay=s["decay"], base=s["base"], window=s["window"])
        return _plain_mass(s)
    # the long sequences stay, as a server keeps its documents; the copies that answers go on from are made and cut down anew
    if own:
        h = s["handle"]
        h.free(s["copies"])
        forked = h.fork(s["rows"], s["copies"])
        status, kept = h.evict(s["base"], s["keep"], s["copies"], recent=s["recent"], first=s["first"], into=s["mass"])
    else:
        _plain_free(c, s["copies"].long(), s["page"])
        forked = _plain_fork(c, s["rows"].long(), s["copies"].long(), s["page"], s["kv_heads"])
        status, kept = _plain_evict(s)
    return forked, status, kept, s["mass"], c["table"], c["lengths"], c["refs"], c["pages"].view(torch.int32)


# ----------------------------------------------------------------------------------------------
# the plain form
# ----------------------------------------------------------------------------------------------
_h = {}


def _hadamard():
    """H_128 by Sylvester's recursion, divided by sqrt(128)."""
    if "h" not in _h:
        h2 = torch.tensor([[1, 1], [1, -1]], dtype=torch.float64)
        _h["h"] = (torch.kron(torch.kron(torch.kron(h2, h2), torch.kron(h2, h2)), torch.kron(h2, torch.kron(h2, h2))) / math.sqrt(D)).to(DEV, torch.float32)
    return _h["h"]


def _views(s):
    """The codes and scales of the pool: [pages, heads, page, 64] bytes and [pages, heads, page, 1 or 2] floats, keys' and values'."""
    page, sf = s["page"], 2 if s["asym"] else 1
    b = s["cache"]["pages"].view(s["cache"]["pages"].shape[0], s["kv_heads"], -1)
    f = b.view(torch.float32)
    a = page * 32
    return (b[..., :page * 64].unflatten(-1, (page, 64)), b[..., page * 64:page * 128].unflatten(-1, (page, 64)),
            f[..., a:a + page * sf].unflatten(-1, (page, sf)), f[..., a + page * sf:a + 2 * page * sf].unflatten(-1, (page, sf)))


def _plain_values(codes, scales, asym):
    """yhat of packed codes and scales, fp32."""
    q = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    if asym:
        return q.float() * scales[..., :1] + scales[..., 1:]
    return ((q ^ 8).to(torch.int8) - 8).float() * scales


def _plain_rows(s, entries, values=True):
    """Keys (and values) of lists of pages [n, m]: [n, kv heads, m * page, 128]."""
    kc, vc, ks, vs = _views(s)
    held = entries.long().clamp(min=0)
    return tuple(_plain_values(b[held], f[held], s["asym"]).transpose(1, 2).flatten(2, 3) for b, f in ((kc, ks), (vc, vs))[:1 + values])


def _plain_queries(s):
    """(query rows, rotated [items, kv heads, group, new tokens, 128]; positions of the tokens [items, new tokens]; which of them there are)"""
    rows, cu, kvh = s["rows"].long(), s["cu"].long(), s["kv_heads"]
    j = torch.arange(s["max_new"], device=DEV)
    count = cu[1:] - cu[:-1]
    q = torch.nn.functional.pad(s["q"].float(), (0, D - s["d"])) @ _hadamard()
    q = q[(cu[:-1, None] + j).clamp(max=s["total"] - 1)].view(len(rows), s["max_new"], kvh, s["heads"] // kvh, D).permute(0, 2, 3, 1, 4)
    return q, s["cache"]["lengths"].long()[rows][:, None] - count[:, None] + j, j < count[:, None]


def _plain_shared(s):
    c, page, rows, kvh = s["cache"], s["page"], s["rows"].long(), s["kv_heads"]
    q, pos, there = _plain_queries(s)
    n, group, mq = len(rows), s["heads"] // kvh, s["max_new"]
    # scores over each group's prefix: its items' rows side by side
    sizes = torch.tensor(s["sizes"], device=DEV)
    item = torch.repeat_interleave(torch.arange(len(sizes), device=DEV), sizes)                  # group of each item
    nth = torch.arange(n, device=DEV) - (sizes.cumsum(0) - sizes)[item]
    prefix = torch.tensor(s["prefix_tokens"], device=DEV)
    most = max(s["prefix_tokens"])
    side = torch.zeros((len(sizes), max(s["sizes"]), kvh, group * mq, D), device=DEV)
    side[item, nth] = q.flatten(2, 3)
    side = side.transpose(1, 2).flatten(2, 3)                                                    # [groups, kv heads, items * group * mq, 128]
    k, v = _plain_rows(s, c["table"][rows[sizes.cumsum(0) - sizes], :most // page])
    score = side @ k.transpose(-1, -2) / math.sqrt(s["d"])
    score = score.masked_fill(torch.arange(score.shape[-1], device=DEV) >= prefix[:, None, None, None], float("-inf"))
    # and over what each item has of its own
    width = -(-s["longest_rest"] // page)
    at = prefix[item][:, None] // page + torch.arange(width, device=DEV)
    k2, v2 = _plain_rows(s, c["table"][rows].gather(1, at.clamp(max=c["table"].shape[1] - 1)))
    score2 = q.flatten(2, 3) @ k2.transpose(-1, -2) / math.sqrt(s["d"])
    t = prefix[item][:, None, None] + torch.arange(width * page, device=DEV)
    seen = (t <= pos[..., None])[:, None, None]                                                  # [items, 1, 1, mq, tokens]
    score2 = score2.unflatten(2, (group, mq)).masked_fill(~seen, float("-inf")).flatten(2, 3)
    top2 = score2.amax(-1, keepdim=True)
    top = score.amax(-1, keepdim=True) if most else torch.full(score.shape[:-1] + (1,), float("-inf"), device=DEV)
    split = lambda x: x.unflatten(2, (max(s["sizes"]), group * mq)).transpose(1, 2)[item, nth]   # noqa: E731    back to items
    both = torch.maximum(top2, split(top))
    both = torch.where(both > float("-inf"), both, 0.0)
    wide = torch.zeros((len(sizes), max(s["sizes"]), kvh, group * mq, 1), device=DEV)
    wide[item, nth] = both
    p = torch.exp(score - wide.transpose(1, 2).flatten(2, 3))
    p2 = torch.exp(score2 - both)
    total = split(p.sum(-1, keepdim=True)) + p2.sum(-1, keepdim=True)
    o = (split(p @ v) + p2 @ v2) / torch.where(total > 0, total, 1.0) @ _hadamard()[:, :s["d"]]
    o = o.unflatten(2, (group, mq)).permute(0, 3, 1, 2, 4).reshape(n, mq, s["heads"], s["d"])
    return o[there].to(torch.bfloat16)


def _plain_mass(s):
    c, page, rows = s["cache"], s["page"], s["rows"].long()
    q, pos, there = _plain_queries(s)
    (k,) = _plain_rows(s, c["table"][rows, :-(-s["longest"] // page)], False)
    score = (q.flatten(2, 3) @ k.transpose(-1, -2) / math.sqrt(s["d"])).unflatten(2, q.shape[2:4])
    length = c["lengths"].long()[rows]
    t = torch.arange(score.shape[-1], device=DEV)
    seen = (t <= pos[..., None]) & (t < length[:, None, None]) & there[..., None]
    if s["window"]:
        seen &= t > pos[..., None] - s["window"]
    seen = seen[:, None, None]
    score = score.masked_fill(~seen, float("-inf"))
    top = score.amax(-1, keepdim=True)
    p = torch.where(seen, torch.exp(score - torch.where(top > float("-inf"), top, 0.0)), 0.0)
    total = p.sum(-1, keepdim=True)
    new = (p / torch.where(total > 0, total, 1.0)).sum((2, 3))[..., :s["longest"]]               # [items, kv heads, tokens]
    t = t[:s["longest"]]
    old = torch.where((t < pos[:, :1])[:, None], s["base"][rows] * s["decay"], 0.0)              # a call's own tokens had nothing before it
    s["mass"][rows] = torch.where((t < length[:, None])[:, None], old + new, s["mass"][rows])
    return s["mass"]


def _held(c, seqs, page):
    """Which entries of these sequences' rows of the table hold pages."""
    return torch.arange(c["table"].shape[1], device=DEV) < ((c["lengths"][seqs] + page - 1) // page)[:, None]


def _plain_free(c, seqs, page):
    ids = c["table"][seqs][_held(c, seqs, page)].long()
    c["refs"].index_add_(0, ids, torch.full_like(ids, -1, dtype=torch.int32))
    c["lengths"][seqs] = 0


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


def _plain_evict(s):
    """The copies keep `keep` tokens: the first ones, the last ones, and for each KV head those with the most weight between; the lower position of two alike."""
    c, page, keep, seqs = s["cache"], s["page"], s["keep"], s["copies"].long()
    length = c["lengths"].long()[seqs]
    t = torch.arange(s["longest"], device=DEV)
    always = (t < s["first"]) | (t >= length[:, None] - s["recent"])
    w = s["base"][seqs].masked_fill(always[:, None], float("inf")).masked_fill((t >= length[:, None])[:, None], -1.0)
    best = torch.sort(w, dim=-1, descending=True, stable=True).indices[..., :keep]
    kept = best.sort(-1).values                                                                  # [items, kv heads, keep]
    if kept.shape[-1] < keep:
        kept = torch.nn.functional.pad(kept, (0, keep - kept.shape[-1]), value=-1)
    cut = length > keep
    short = torch.arange(keep, device=DEV)
    kept = torch.where(cut[:, None, None], kept, torch.where(short < length[:, None], short, -1)[:, None])
    weight = s["base"][seqs].gather(-1, kept.clamp(min=0))
    s["mass"][seqs, :, :weight.shape[-1]] = torch.where(kept >= 0, weight, s["mass"][seqs, :, :weight.shape[-1]])
    # pages of their own for what stays, the lowest free ones in the items' order
    need = -(-keep // page)
    at = torch.nonzero(cut)[:, 0]
    ids = torch.nonzero(c["refs"] == 0)[:, 0][:len(at) * need].view(len(at), need)
    token = kept[at]                                                                             # [cut items, kv heads, keep]
    old = c["table"][seqs[at]].long().gather(1, (token // page).flatten(1)).view(token.shape)
    head = torch.arange(s["kv_heads"], device=DEV)[:, None]
    new = ids[:, short // page][:, None].expand(token.shape)
    for x in _views(s):
        x[new, head, short % page] = x[old, head, token % page]
    gone = c["table"][seqs[at]][_held(c, seqs[at], page)].long()
    c["refs"].index_add_(0, gone, torch.full_like(gone, -1, dtype=torch.int32))
    c["refs"][ids] = 1
    c["table"][seqs[at], :need] = ids.to(torch.int32)
    c["lengths"][seqs[at]] = keep
    return torch.zeros(len(seqs), dtype=torch.int32, device=DEV), kept.to(torch.int32)


# ----------------------------------------------------------------------------------------------
# the definition in 64 bits, one sequence at a time and in the rows' own basis
# ----------------------------------------------------------------------------------------------
def _signs():
    i = torch.arange(D, device=DEV)
    x = i[:, None] & i[None, :]
    parity = sum((x >> b) & 1 for b in range(7)) % 2
    return 1.0 - 2.0 * parity.double()


def _exact_rows(s, seq, count, which):
    """The first `count` cached tokens of a sequence as rows of their own basis: [kv heads, count, d], keys (0) or values (1)."""
    c, page, sf = s["cache"], s["page"], 2 if s["asym"] else 1
    ids = c["table"][seq, :-(-count // page)].long()
    blocks = c["pages"][ids].view(len(ids), s["kv_heads"], -1)
    codes = blocks[:, :, which * page * 64:(which + 1) * page * 64].reshape(len(ids), s["kv_heads"], page, 64)
    at = page * 128 + which * page * 4 * sf
    scales = blocks[:, :, at:at + page * 4 * sf].contiguous().view(torch.float32).reshape(len(ids), s["kv_heads"], page, sf).double()
    y = torch.empty(codes.shape[:3] + (D,), dtype=torch.float64, device=DEV)
    y[..., 0::2], y[..., 1::2] = (codes % 16).double(), (codes // 16).double()
    y = y * scales[..., :1] + scales[..., 1:] if s["asym"] else (y - 16 * (y > 7)) * scales
    return (y.movedim(1, 0).flatten(1, 2)[:, :count] @ _signs() / D ** 0.5)[..., :s["d"]]


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "evict":                                  # the weights that stay; the others are whole numbers, and bytes that move
        out = s["mass"].double().cpu().numpy()
        base, keep = s["base"].cpu().numpy(), case["keep"]
        for dst, src in zip(s["copies"].tolist(), s["rows"].tolist()):
            length = int(s["cache"]["lengths"][src])
            for h in range(case["kv_heads"]):
                stay = np.arange(length)
                if length > keep:
                    a, b = s["first"], length - s["recent"]
                    order = np.lexsort((np.arange(a, b), -base[dst, h, a:b].astype(np.float64)))[:keep - a - s["recent"]]
                    stay = np.sort(np.concatenate([stay[:a], a + order, stay[b:]]))
                out[dst, h, :len(stay)] = base[dst, h, stay]
        return None, None, None, torch.from_numpy(out), None, None, None, None
    kvh, group, d = case["kv_heads"], case["heads"] // case["kv_heads"], case["d"]
    cu, rows, lengths = s["cu"].tolist(), s["rows"].tolist(), s["cache"]["lengths"].tolist()
    mass = case["kind"] == "mass"
    out = torch.zeros(s["mass"].shape if mass else s["q"].shape, dtype=torch.float64, device=DEV)
    for i, seq in enumerate(rows):
        count, length = cu[i + 1] - cu[i], lengths[seq]
        k = _exact_rows(s, seq, length, 0)
        v = None if mass else _exact_rows(s, seq, length, 1)
        if mass:
            out[seq, :, :length - count] = s["base"][seq, :, :length - count].double() * case["decay"]
        for a in range(0, count, 128):                           # some query tokens at a time
            b = min(count, a + 128)
            q = s["q"][cu[i] + a:cu[i] + b].double().view(b - a, kvh, group, d)
            score = torch.einsum("qhgd,hkd->qhgk", q, k) / d ** 0.5
            far = (length - count + torch.arange(a, b, device=DEV))[:, None] - torch.arange(length, device=DEV)
            hidden = (far < 0) | (far >= case["window"]) if mass and case["window"] else far < 0
            p = torch.softmax(score.masked_fill(hidden[:, None, None], -math.inf), -1)
            if mass:
                out[seq, :, :length] += p.sum((0, 2))
            else:
                out[cu[i] + a:cu[i] + b] = torch.einsum("qhgk,hkd->qhgd", p, v).reshape(b - a, case["heads"], d)
    return out


# ----------------------------------------------------------------------------------------------
# what a pass cannot do without
# ----------------------------------------------------------------------------------------------
def work(case):
    kind, sf, kvh = case["kind"], 2 if case["asym"] else 1, case["kv_heads"]
    token = 128 + 8 * sf                                         # bytes of a token and KV head in the cache
    if kind == "shared":
        sizes, prefix, rest, new = _family(case)
        read, pairs, i = 0, 0, 0
        for size, p in zip(sizes, prefix):
            read += p + sum(rest[i:i + size])
            pairs += sum(b * (p + r - b) + b * (b + 1) // 2 for r, b in zip(rest[i:i + size], new[i:i + size]))
            i += size
        return {"bytes": read * kvh * token + 2 * 2 * sum(new) * case["heads"] * case["d"], "flops": 4 * 128 * case["heads"] * pairs}
    kv, new = _lengths(case)
    if kind == "mass":
        window, pairs, read = case["window"], 0, 0
        for a, b in zip(kv, new):
            pairs += sum(min(window, a - b + j + 1) for j in range(b)) if window else b * (a - b) + b * (b + 1) // 2
            read += min(a, window + b - 1) if window else a
        # keys of the tokens that are seen, weights of all: those before the call's own are read where they count
        return {"bytes": kvh * (read * token // 2 + 4 * sum(kv) + (4 * sum(a - b for a, b in zip(kv, new)) if case["decay"] else 0))
                + 2 * sum(new) * case["heads"] * case["d"], "flops": 2 * 128 * case["heads"] * pairs}
    keep, page = case["keep"], case["page"]
    cut = [v for v in kv if v > keep]
    # weights looked through, the kept tokens read and written, their positions and weights, the table and the counters of shared pages
    return {"bytes": kvh * (4 * sum(cut) + len(cut) * keep * (2 * token + 4 + 4)) + 16 * sum(-(-v // page) for v in kv), "flops": 0}
