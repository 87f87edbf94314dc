"""How far a row of attention over the paged KV cache may be from the formula in 64 bits, in its Euclidean norm.

kv_util.attention bounds every element by the worst case, in which all roundings of a row pull the same way; for long sequences that is more than the
result itself.  Here roundings count as what they are, independent of one another: a number that is rounded to a type with half steps u (relative to it) is
off by at most u and by u / sqrt(3) in the root mean square, so the result's error, a sum of such, has the variance

    V = sum_j p_j^2 [ (W^2 / 3) |u_j|^2 + S_j^2 |v_j - o|^2 + R_j ]

with W = 2^-11 the half step of a weight, u_j what it multiplies, S_j the deviation of token j's score and R_j that of its value row:
  few rows (up to 16)   u = v - mid (the middle, mid = lo + 8 Delta, 0 for a symmetric plan, is weighted in 32 bits); a query coordinate is rounded to 1 / 65024 of the row's largest, m: S_j^2 = scale^2 (m / 65024)^2 / 3 |k_j|^2, R_j = 0;
  many rows             u = v; query coordinates, Delta, mid and the coordinates that they give are fp16:
                        S_j^2 = scale^2 W^2 / 3 (2 sum_i q_i^2 k_i^2 + (q . (k - mid))^2 + (q . mid)^2), R_j = W^2 / 3 (|v|^2 + |v - mid|^2 + 128 mid^2).
Sums in 24 bits and ex2 add 2^-20 of sums of absolute values.  The norm of such an error stays within six deviations (a sum of bounded independent terms is
past them with a probability of 2 e^-18), and bf16 rounds the result by at most 2^-8 of itself:

    |got - o| <= 2^-8 |o| + 6 sqrt(V) + 2^-20 sum_j p_j |v_j|.
"""
import torch

W = 2.0 ** -11


def attend(x, k, km, v, vm, seen, scale, few):
    """x [tokens, kv heads, group, 128] rotated queries; k, v [kv heads, cached, 128] and their middles [kv heads, cached]; seen [tokens, cached].
    Returns the rotated result o and the bound on the norm of its error [tokens, kv heads, group]."""
    s = torch.einsum("qhgd,hkd->qhgk", x, k) * scale
    s = s.masked_fill(~seen[:, None, None], float("-inf"))
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top == float("-inf"), torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    p = torch.where(total == 0, torch.zeros_like(p), p / total)
    o = torch.einsum("qhgk,hkd->qhgd", p, v)
    v2 = v.square().sum(-1)[None, :, None]
    apart = (v2 - 2 * torch.einsum("qhgd,hkd->qhgk", o, v) + o.square().sum(-1, keepdim=True)).clamp(min=0)
    if few:
        dev = (scale / 65024) ** 2 / 3 * x.abs().amax(-1, keepdim=True).square() * k.square().sum(-1)[None, :, None]
        rows, u2 = torch.zeros_like(v2), (v - vm[..., None]).square().sum(-1)[None, :, None]
    else:
        mid = x.sum(-1, keepdim=True) * km[None, :, None]
        both = torch.einsum("qhgd,hkd->qhgk", x.square(), k.square())
        dev = scale ** 2 * W ** 2 / 3 * (2 * both + (torch.einsum("qhgd,hkd->qhgk", x, k) - mid).square() + mid.square())
        vm2, u2 = 128 * vm.square()[None, :, None], v2
        rows = W ** 2 / 3 * (v2 + (v - vm[..., None]).square().sum(-1)[None, :, None] + vm2)
    var = (p.square() * (W ** 2 / 3 * u2 + dev * apart + rows)).sum(-1)
    bound = 2.0 ** -8 * o.norm(dim=-1) + 6 * var.sqrt() + 2.0 ** -20 * (p * v2.sqrt()).sum(-1)
    return o, bound


def seen_by(length, count, causal, window, device):
    pos = (length - count + torch.arange(count, device=device))[:, None]
    t = torch.arange(length, device=device)
    seen = (t <= pos) if causal else (t < length) & (pos > -length - count)
    return seen & (t > pos - window) if window else seen


def check(cache, got, q, seqs, counts, causal=True, window=0, scale=0.0):
    """The call's rows against the formula, by their norms; returns the largest of error / bound."""
    import kv_util
    d, kvh = cache.plan.info.d, cache.n_kv_heads
    heads = q.shape[1]
    group, few = heads // kvh, max(counts) * (heads // kvh) <= 16
    h = kv_util.h128()[:, :d] / 128 ** 0.5
    worst, at = 0.0, 0
    for seq, count in zip(seqs, counts):
        length = int(cache.lengths[seq])
        if length == 0:
            assert not got[at:at + count].any()
            at += count
            continue
        k, v, km, vm = kv_util.rows_of(cache, seq, middles=True)
        # middles keep their sign here
        if cache.plan.info.asymmetric:
            km, vm = signed_middles(cache, seq, length)
        for a in range(0, count, 128):
            b = min(count, a + 128)
            y = got[at + a:at + b].double()
            x = torch.einsum("qhd,cd->qhc", q[at + a:at + b].double(), h).view(b - a, kvh, group, 128)
            o, bound = attend(x, k, km, v, vm, seen_by(length, count, causal, window, q.device)[a:b], scale or d ** -0.5, few)
            off = (y - (o.reshape(b - a, heads, 128) @ h)).norm(dim=-1)
            ratio = (off / bound.reshape(b - a, heads).clamp(min=1e-300))
            assert bool((ratio <= 1).all()), ("sequence %d of %d tokens, %d queries" % (seq, length, count), (~(ratio <= 1)).nonzero()[:8].tolist(), float(ratio.max()))
            worst = max(worst, float(ratio.max()))
        at += count
    return worst


def signed_middles(cache, seq, length):
    ps = cache.page_size
    ids = cache.page_table[seq, :-(-length // ps)].long()
    blocks = cache.pages[ids].view(len(ids), cache.n_kv_heads, -1)
    out = []
    for i in range(2):
        at = ps * 128 + i * ps * 8
        s = blocks[:, :, at:at + ps * 8].contiguous().view(torch.float32).reshape(len(ids), cache.n_kv_heads, ps, 2).double()
        out.append((s[..., 1] + 8 * s[..., 0]).transpose(0, 1).flatten(1, 2)[:, :length])
    return out
