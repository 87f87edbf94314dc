"""The ring of k_kv_attn_few: a warp reads a stage when the copy into it has ended, however late single copies are.

On the CPU a model of the ring's barriers with the sizes of the source; on the GPU first calls on pools that nothing has touched, where copies are slow."""
import os
import random
import re

import pytest
import torch

import kv_norms
from kv_util import DEV, filled

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2504_13989_b200", "csrc", "gbs_kv_attn.cu")


class Barrier:
    """A wait for a parity passes when the current phase has the other one: it knows nothing of phases further back."""

    def __init__(self):
        self.ended = 0

    def passes(self, parity):
        return (self.ended & 1) != parity


def run_ring(warps, stages, units, rng):
    """One block's units; every step some role that can go on does.  Returns what went wrong first, or None."""
    full, empty = [Barrier() for _ in range(stages)], [Barrier() for _ in range(stages)]
    holds, flying, sent, unit = [None] * stages, set(), 0, list(range(warps))
    slow = set(rng.sample(range(units), max(1, units // 15)))
    while any(u < units for u in unit):
        can = [("warp", w) for w in range(warps) if unit[w] < units and full[unit[w] % stages].passes((unit[w] // stages) & 1)]
        if sent < units and all(u // stages == 0 or empty[u % stages].passes((u // stages - 1) & 1) for u in range(sent, min(sent + 4, units))):
            can.append(("send", 0))
        fast = [u for u in flying if u not in slow]
        can += [("land", u) for u in fast]
        if not can or rng.random() < 0.02:
            can += [("land", u) for u in flying]
        if not can:
            return "nobody can go on"
        what, i = rng.choice(can)
        if what == "send":
            for u in range(sent, min(sent + 4, units)):
                if any(v % stages == u % stages for v in flying):
                    return "unit %d is sent for while another is on its way into its stage" % u
                flying.add(u)
            sent = min(sent + 4, units)
        elif what == "land":
            flying.remove(i)
            holds[i % stages] = i
            full[i % stages].ended += 1
        else:
            u = unit[i]
            if holds[u % stages] != u or u in flying:
                return "warp %d reads unit %d before it is there" % (i, u)
            empty[u % stages].ended += 1
            unit[i] += warps
    return None


def sizes():
    text = open(SOURCE).read()
    return tuple(int(re.search(r"constexpr int %s = (\d+)" % name, text).group(1)) for name in ("WARPS", "STAGES"))


def test_a_unit_is_read_when_it_is_there():
    warps, stages = sizes()
    for seed in range(300):
        rng = random.Random(seed)
        assert run_ring(warps, stages, rng.randrange(1, 200), rng) is None


def test_the_model_tells_rings_whose_stages_change_warps():
    """Eleven stages for four warps: a warp two units ahead of its neighbour reads what is not there."""
    found = {run_ring(4, 11, 150, random.Random(seed)) for seed in range(50)}
    assert any(f is not None for f in found)


@pytest.mark.gpu
@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("lengths,heads,kv_heads,page", [([3000, 70, 20000] * 60, 2, 2, 32), ([60000, 20011], 16, 2, 64), ([900] * 64, 8, 8, 16)])
def test_first_calls_on_new_pools(lengths, heads, kv_heads, page, asym):
    from paper_2504_13989_b200 import Plan
    from paper_2504_13989_b200 import build as gbs_build
    gbs_build.build()
    with Plan(128, 128, 1, 4, 128, 0.9, asymmetric=asym) as plan:
        gen = torch.Generator(device=DEV)
        gen.manual_seed(7)
        n = len(lengths)
        q = torch.randn((n, heads, 128), generator=gen, device=DEV).to(torch.bfloat16)
        for rep in range(10):
            torch.cuda.empty_cache()
            cache = filled(plan, lengths, kv_heads, page, seed=rep)
            torch.empty(1 << 28, dtype=torch.uint8, device=DEV).fill_(rep)      # nothing of the pool is left in the cache on the chip
            torch.cuda.synchronize()
            first = cache.attention(q)
            assert all(torch.equal(cache.attention(q), first) for _ in range(3))
            if rep < 2:
                kv_norms.check(cache, first, q, range(n), [1] * n)
        assert plan.device_status() == 0
