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
