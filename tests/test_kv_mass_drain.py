"""What a block of the weights' second pass for many rows waits for before it ends early: the copies of query rows that it has sent for, whatever came of them.

A model of the two buffers' barriers on the CPU, with the counts that the source waits by."""
import os
import random
import re

import pytest

from test_kv_ring import Barrier

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2504_13989_b200", "csrc", "gbs_tc_kvmass.cu")


def counts():
    """The expressions by which the two buffers are waited for."""
    text = open(SOURCE).read()
    found = {int(b): e for b, e in re.findall(r"drain_copies\(&S\.qfull\[(\d)\], 1, \(int\)(.+?)\);", text)}
    assert sorted(found) == [0, 1]
    return found


def ends_early(segments, expressions, rng):
    """Segments of one or two tiles; the fetching warp goes ahead until another role gives up, at any time.  Whether a wait then passes while a copy is on its way."""
    full, free = [Barrier(), Barrier()], [Barrier(), Barrier()]
    n = {"used": 0, "used1": 0, "sent": 0, "sent1": 0}
    flying = set()
    at, tile = 0, 0
    taken = [0, 0]                               # fillings that the others have done with
    for _ in range(rng.randrange(1, 12 * len(segments))):
        can = [("land", b) for b in flying] + [("take", b) for b in (0, 1) if full[b].ended > taken[b]]
        if at < len(segments):
            filled = n["used1"] if tile else n["used"]
            if filled == 0 or free[tile].passes((filled - 1) & 1):
                can.append(("send", tile))
        if not can:
            break
        what, b = rng.choice(can)
        if what == "land":
            flying.remove(b)
            full[b].ended += 1
        elif what == "take":
            taken[b] += 1
            free[b].ended += 1
        else:
            assert b not in flying
            flying.add(b)
            n["sent1" if b else "sent"] += 1
            tile += 1
            if tile == segments[at]:
                n["used"] += 1
                n["used1"] += segments[at] > 1
                at, tile = at + 1, 0
    # a wait for so many copies is one for the phase of the last of them
    return any(count > 0 and b in flying and full[b].passes((count - 1) & 1) for b, count in ((b, eval(e, {}, dict(n))) for b, e in expressions.items())) or \
        any(b in flying and eval(expressions[b], {}, dict(n)) <= 0 for b in (0, 1))


def trials(expressions):
    for seed in range(2000):
        rng = random.Random(seed)
        yield ends_early([rng.choice([1, 2]) for _ in range(rng.randrange(1, 9))], expressions, rng)


def test_a_block_ends_after_its_copies():
    assert not any(trials(counts()))


@pytest.mark.parametrize("expressions", [{0: "used + 1", 1: "used1 + 1"}, {0: "used", 1: "used1"}])
def test_the_model_tells_counts_of_segments(expressions):
    assert any(trials(expressions))
