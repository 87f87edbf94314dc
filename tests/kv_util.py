"""A paged KV cache in plain Python and 64 bits: the pool's bookkeeping as lists, its rows and attention over them as formulas."""
import numpy as np
import scipy.linalg
import torch

DEV = "cuda:0"
H = scipy.linalg.hadamard(128).astype(np.float64)


def h128():
    return torch.from_numpy(H).to(DEV)


def rows_of(cache, seq, count=None, middles=False):
    """Keys and values [heads, tokens, 128] (rotated domain, 64 bits) that the first `count` tokens of a sequence stand for; with `middles`, behind
    them |lo + 8 Delta| of their rows [heads, tokens] (0 for a symmetric plan)."""
    ps, asym = cache.page_size, bool(cache.plan.info.asymmetric)
    sf = 2 if asym else 1
    count = int(cache.lengths[seq]) if count is None else count
    ids = cache.page_table[seq, :-(-count // ps)].long()
    blocks = cache.pages[ids].view(len(ids), cache.n_kv_heads, -1)
    out, mid = [], []
    for i in range(2):
        c = blocks[:, :, i * ps * 64:(i + 1) * ps * 64].reshape(len(ids), cache.n_kv_heads, ps, 64).to(torch.int16)
        q = torch.stack([c & 15, c >> 4], -1).flatten(-2)
        at = ps * 128 + i * ps * 4 * sf
        s = blocks[:, :, at:at + ps * 4 * sf].contiguous().view(torch.float32).reshape(len(ids), cache.n_kv_heads, ps, sf).double()
        q = q.double()
        y = q * s[..., :1] + s[..., 1:] if asym else (q - 16 * (q > 7)) * s
        out.append(y.transpose(0, 1).flatten(1, 2)[:, :count])
        mid.append(((s[..., 1] + 8 * s[..., 0]).abs() if asym else 0 * s[..., 0]).transpose(0, 1).flatten(1, 2)[:, :count])
    return out + mid if middles else out


def attention(cache, q, seqs, cu, causal=True, window=0, scale=0.0, max_len=0, few=True):
    """(result, tolerance) in 64 bits for the rows of the items; the others are NaN.

    The tolerance, with e the error of a score: the result is a mean of rows vhat with weights p, each off by a factor of at most 1 + 2 e + r
    (numerator and denominator; r: the rounding of the probabilities and of the sums), so off by at most (2 e + r) max|vhat|_2 in any
    coordinate of any basis, and then rounded to bf16 (2^-8 of itself).  e <= scale |q|_2 |khat|_2 (b + 128 2^-23): the query row is rounded to
    1 / 65024 of its largest coordinate in each of 128 places (few rows: at most sqrt(128) / 65024 of its norm), or to 11 bits of each coordinate
    (2^-12, and sqrt(128) 2^-24 for what falls below fp16's normal numbers); 128 products are added up in 24 bits.  A probability is rounded to
    11 bits (2^-11: 2^-12, and as much for ex2, log2 and the sums).

    With many rows cached rows are rounded too: a coordinate x = c Delta + mid, mid = lo + 8 Delta (symmetric: 0), has Delta, mid and then x itself
    rounded to 11 bits, so it is off by at most 2^-12 (|x - mid| + |mid| + |x|) <= 2^-11 (|x| + |mid|), a row by 2^-11 (|x|_2 + sqrt(128) |mid|)
    =: 2^-11 (|x|_2 + m).  That adds scale |q|_2 2^-11 (|khat|_2 + m) to e, and 2^-11 max(|vhat|_2 + m) to the result.
    """
    d = cache.plan.info.d
    heads, kvh = q.shape[1], cache.n_kv_heads
    group = heads // kvh
    want = torch.full(q.shape, float("nan"), dtype=torch.float64, device=q.device)
    tol = torch.full(q.shape, float("nan"), dtype=torch.float64, device=q.device)
    scale = scale or d ** -0.5
    b = 128 ** 0.5 / 65024 if few else 2.0 ** -12 + 128 ** 0.5 * 2.0 ** -24
    r = 2.0 ** -11
    for i, seq in enumerate(seqs):
        length, count = int(cache.lengths[seq]), cu[i + 1] - cu[i]
        if count == 0:
            continue
        x = torch.zeros((count, heads, 128), dtype=torch.float64, device=q.device)
        x[..., :d] = q[cu[i]:cu[i + 1]].double()
        x = (x @ h128() / 128 ** 0.5).view(count, kvh, group, 128)
        if length == 0:
            want[cu[i]:cu[i + 1]], tol[cu[i]:cu[i + 1]] = 0, 0
            continue
        k, v, km, vm = rows_of(cache, seq, middles=True)
        s = torch.einsum("qhgd,hkd->qhgk", x, k) * scale
        pos = (length - count + torch.arange(count, device=q.device))[:, None]
        t = torch.arange(length, device=q.device)
        seen = (t <= pos) if causal else (t < length) & (pos > -length - count)
        if window:
            seen = seen & (t > pos - window)
        if max_len:
            seen = seen & (t < max_len)
        s = s.masked_fill(~seen[:, None, None], float("-inf"))
        top = s.amax(-1, keepdim=True)
        p = torch.exp(s - torch.where(top == float("-inf"), torch.zeros_like(top), top))
        total = p.sum(-1, keepdim=True)
        p = torch.where(total == 0, torch.zeros_like(p), p / total)
        o = torch.einsum("qhgk,hkd->qhgd", p, v) @ h128()[:, :d] / 128 ** 0.5
        kn = (k.norm(dim=-1)[None] * seen[:, None]).amax(-1)
        vn = (v.norm(dim=-1)[None] * seen[:, None]).amax(-1)
        e = abs(scale) * x.norm(dim=-1) * kn[:, :, None] * (b + 128 * 2.0 ** -23)
        lim = 2.0 ** -8 * o.abs() + ((2 * e + r) * vn[:, :, None])[..., None]
        if not few:
            kr, vr = (2.0 ** -11 * ((y.norm(dim=-1) + 128 ** 0.5 * m)[None] * seen[:, None]).amax(-1) for y, m in ((k, km), (v, vm)))
            lim = lim + (2 * abs(scale) * x.norm(dim=-1) * kr[:, :, None] * vn[:, :, None] + vr[:, :, None])[..., None]
        want[cu[i]:cu[i + 1]] = o.reshape(count, heads, d)
        tol[cu[i]:cu[i + 1]] = lim.reshape(count, heads, d)
    return want, tol


class Model:
    """The bookkeeping of a pool as lists."""

    def __init__(self, n_pages, page_size, n_seqs, max_pages):
        self.ps, self.max_pages, self.n_seqs = page_size, max_pages, n_seqs
        self.refs = [0] * n_pages
        self.pages = [[] for _ in range(n_seqs)]
        self.lengths = [0] * n_seqs
        self.copies = []                                     # (page, page, tokens) that forks copied

    def _serve(self, wishes):
        """wishes: (status, need) per item -> the pages of each; None: refused"""
        free, before, got = [p for p, r in enumerate(self.refs) if r == 0], 0, []
        for status, need in wishes:
            if status != 0:
                got.append(None)
                continue
            got.append(free[before:before + need] if before + need <= len(free) or need == 0 else None)
            before += need
        for pages in got:
            for p in pages or []:
                self.refs[p] = 1
        return got

    def extend(self, seqs, counts):
        seen, wishes = set(), []
        for s, c in zip(seqs, counts):
            if not 0 <= s < self.n_seqs:
                wishes.append((1, 0))
                continue
            if s in seen:
                wishes.append((5, 0))
                continue
            seen.add(s)
            if c < 0:
                wishes.append((1, 0))
            elif self.lengths[s] + c > self.max_pages * self.ps:
                wishes.append((4, 0))
            else:
                wishes.append((0, -(-(self.lengths[s] + c) // self.ps) - len(self.pages[s])))
        got, status = self._serve(wishes), []
        for s, c, (st, _), pages in zip(seqs, counts, wishes, got):
            if st == 0 and pages is not None:
                self.pages[s] += pages
                self.lengths[s] += c
            status.append(st if st else (0 if pages is not None else 3))
        return status

    def fork(self, src, dst):
        seen, wishes = set(), []
        was = [(n, list(p)) for n, p in zip(self.lengths, self.pages)]
        for a, b in zip(src, dst):
            if not 0 <= b < self.n_seqs:
                wishes.append((1, 0))
            elif b in seen:
                wishes.append((5, 0))
            elif not 0 <= a < self.n_seqs:
                seen.add(b)
                wishes.append((1, 0))
            else:
                seen.add(b)
                wishes.append((2, 0) if was[b][0] else (0, int(was[a][0] % self.ps != 0)))
        got, status = self._serve(wishes), []
        for a, b, (st, need), pages in zip(src, dst, wishes, got):
            if st == 0 and pages is not None:
                n, held = was[a]
                full = n // self.ps
                for p in held[:full]:
                    self.refs[p] += 1
                if need:
                    self.copies.append((held[full], pages[0], n % self.ps))
                self.pages[b] = held[:full] + pages
                self.lengths[b] = n
            status.append(st if st else (0 if pages is not None else 3))
        return status

    def free(self, seqs):
        for s in seqs:
            if 0 <= s < self.n_seqs:
                for p in self.pages[s]:
                    self.refs[p] -= 1
                self.pages[s], self.lengths[s] = [], 0

    def check(self, cache):
        assert cache.lengths.tolist() == self.lengths
        assert cache.refs.tolist() == self.refs
        table = cache.page_table.tolist()
        for s in range(self.n_seqs):
            assert table[s][:len(self.pages[s])] == self.pages[s], s


def filled(plan, lengths, n_kv_heads, page_size, seed=0, spare=3, scale=1.0):
    """A pool whose sequences hold random rows, their pages in no order; every float of the pool that no token has is a NaN."""
    from paper_2504_13989_b200 import KVCache
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    need = [-(-n // page_size) for n in lengths]
    n_pages = sum(need) + spare
    cache = KVCache.create(plan, n_pages, n_kv_heads, page_size, len(lengths), max(need) + 1, DEV)
    order = torch.randperm(n_pages, generator=gen, device=DEV).tolist()
    at = 0
    cache.pages.random_(0, 256, generator=gen)
    for s, n in enumerate(need):
        if n:
            cache.page_table[s, :n] = torch.tensor(order[at:at + n], dtype=torch.int32, device=DEV)
            cache.refs[cache.page_table[s, :n].long()] = 1
        at += n
    sf = 2 if plan.info.asymmetric else 1
    cache.pages.view(torch.float32).view(n_pages, n_kv_heads, -1)[..., page_size * 32:page_size * (32 + 2 * sf)] = float("nan")
    cache.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
    total = sum(lengths)
    if total:
        k = (torch.randn((total, n_kv_heads, plan.info.d), generator=gen, device=DEV) * scale).to(torch.bfloat16)
        v = torch.randn((total, n_kv_heads, plan.info.d), generator=gen, device=DEV).to(torch.bfloat16)
        cu = torch.tensor([0] + lengths, device=DEV).cumsum(0).to(torch.int32)
        cache.append(k, v, None, cu)
    return cache
