"""KVCache's calls on a stream of their own, with work on the caller's stream that is not waited for."""
import pytest
import torch

from kv_util import DEV, filled
from paper_2504_13989_b200 import Plan
from paper_2504_13989_b200 import build as gbs_build

pytestmark = pytest.mark.gpu


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def test_results_lie_in_memory_that_no_waiting_work_writes():
    """A block that was let go on the caller's stream is still to be written there when the call on the other stream runs."""
    gbs_build.build()
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = filled(plan, [4000], 2, 64, seed=3)
        q = torch.randn((4000, 16, 128), device=DEV).to(torch.bfloat16)
        cu, seqs, side = ints(0, 4000), ints(0), torch.cuda.Stream()
        want = cache.attention(q, seqs, cu, 4000)
        rows = cache.read(seqs, cu, 4000)
        torch.cuda.synchronize()
        for _ in range(3):
            torch.cuda.empty_cache()
            blocks = [torch.empty_like(t) for t in (want, *rows)]
            torch.cuda.synchronize()
            torch.cuda._sleep(100_000_000)
            for b in blocks:
                b.fill_(float("nan"))
            del b, blocks
            got = cache.attention(q, seqs, cu, 4000, stream=side)
            k, v = cache.read(seqs, cu, 4000, stream=side)
            torch.cuda.synchronize()
            assert torch.equal(got, want) and torch.equal(k, rows[0]) and torch.equal(v, rows[1])


def test_two_divided_calls_at_the_same_time():
    """Both calls' long axes are split and joined, each through a workspace of its own."""
    gbs_build.build()
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = filled(plan, [30000, 7000], 4, 64, seed=5)
        side = torch.cuda.Stream()
        for count in (1, 40):
            qs = [torch.randn((2 * count, 16, 128), device=DEV).to(torch.bfloat16) for _ in range(2)]
            cu = ints(0, count, 2 * count)
            want = [cache.attention(q, None, cu, count) for q in qs]
            torch.cuda.synchronize()
            for _ in range(10):
                got = []
                for _ in range(4):
                    got.append(cache.attention(qs[0], None, cu, count))
                    got.append(cache.attention(qs[1], None, cu, count, stream=side))
                torch.cuda.synchronize()
                assert all(torch.equal(g, want[i & 1]) for i, g in enumerate(got))
        assert plan.device_status() == 0


def test_captured_calls_that_are_given_a_stream():
    """The capturing stream itself, and one that forks from it and joins it again."""
    gbs_build.build()
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = filled(plan, [3000, 700, 40], 4, 64, seed=6)
        seqs, cu = ints(2, 0, 1), ints(0, 1, 41, 42)
        q = torch.randn((42, 16, 128), device=DEV).to(torch.bfloat16)
        side = torch.cuda.Stream()
        one, none = ints(2), ints(0)
        cache.attention(q, seqs, cu, 40), cache.read(seqs, cu, 42), cache.extend(one, none)
        torch.cuda.synchronize()
        for fork in (False, True):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                s = torch.cuda.current_stream()
                if fork:
                    side.wait_stream(s)
                    s = side
                got = cache.attention(q, seqs, cu, 40, stream=s)
                rows = cache.read(seqs, cu, 42, stream=s)
                status = cache.extend(one, none, stream=s)
                if fork:
                    torch.cuda.current_stream().wait_stream(side)
            for _ in range(3):
                q.copy_(torch.randn_like(q))
                g.replay()
                assert status.tolist() == [0] and torch.equal(got, cache.attention(q, seqs, cu, 40))
                assert all(torch.equal(a, b) for a, b in zip(rows, cache.read(seqs, cu, 42)))
