"""What attention over shared prefixes does when one of its bounded waits runs out, in the pass over what groups share and in the one over what is an item's own:
the kernels end, the code stands in the plan's status word, and nothing is written but rows of the result and the workspace.  gbs_selftest_kv_shared_attention
makes the waits run out; nothing faults or hangs."""
import ctypes

import pytest
import torch

from paper_2504_13989_b200 import Plan, binding
from paper_2504_13989_b200 import build as gbs_build
from kv_util import DEV
from test_gpu_kv_shared import LONG, check, cu_of, forked, ints, rows
from test_kv_host import INVALID, OK, P, plan, pool

GUARD = 1 << 20
FEW, MANY = (61, 62, 63, 64), (71, 72, 73, 74, 75, 76, 77)


@pytest.fixture(scope="module", autouse=True)
def built():
    gbs_build.build()


def test_refusals():
    lib, c = binding.lib(), pool()

    def f(code, segment, n=2, flags=1, q=P):
        return lib.gbs_selftest_kv_shared_attention(plan(), ctypes.byref(c), P, P, n, 3, 2, P, 1, 0, 0, q, 1024, 128, 8, 0.0, flags, P + 4096, 1024, 128, P, 1 << 40, code,
                                                    segment, None)
    for code in (0, 1, -1, 60, 65, 70, 78, 81, 99, 1 << 20):
        assert f(code, 0) == INVALID
    assert f(61, -1) == INVALID and f(61, 0, flags=2) == INVALID and f(61, 0, q=None) == INVALID and f(64, 3, n=0) == OK


class Call:
    """One call on prompts with as many forks each, its result and workspace between guards."""

    def __init__(self, prompts, forks, own, count, asym):
        self.plan = Plan(128, 128, 1, 4, 128, 0.9, asymmetric=asym)
        n = len(prompts) * forks
        self.cache = forked(self.plan, prompts, [i // forks for i in range(n)], [own + i % 7 for i in range(n)], 2, 32)
        self.n, self.count, self.groups = n, count, len(prompts)
        self.q = rows(n * count, 4, 128, 5)
        self.seqs, self.cu, self.cuts = ints(range(len(prompts), len(prompts) + n)), ints(cu_of([count] * n)), ints(range(0, n + 1, forks))
        self.out = torch.full((2 * GUARD + self.q.numel(),), 7.0, dtype=torch.bfloat16, device=DEV)
        need = ctypes.c_int64(0)
        assert binding.lib().gbs_kv_shared_attention_workspace(self.plan.handle, ctypes.byref(self.cache._c), n, n * count, count, self.groups, LONG, 4, ctypes.byref(need)) == OK
        self.need = need.value
        self.work = torch.full((2 * GUARD + (self.need + 15) // 16 * 16,), 77, dtype=torch.uint8, device=DEV)
        self.kept = [t.clone() for t in self.cache._kept + (self.q, self.cu, self.cuts, self.seqs)]

    def run(self, code=None, segment=0):
        args = [self.plan.handle, ctypes.byref(self.cache._c), self.seqs.data_ptr(), self.cu.data_ptr(), self.n, self.n * self.count, self.count, self.cuts.data_ptr(),
                self.groups, 0, LONG, self.q.data_ptr(), 512, 128, 4, 0.0, 1, self.out.data_ptr() + 2 * GUARD, 512, 128, self.work.data_ptr() + GUARD, self.need]
        if code is None:
            assert binding.lib().gbs_kv_shared_attention(*args, None) == OK
        else:
            assert binding.lib().gbs_selftest_kv_shared_attention(*args, code, segment, None) == OK
        torch.cuda.synchronize()
        inner = self.out[GUARD:-GUARD].clone()
        self.out[GUARD:-GUARD] = 7.0
        assert bool((self.out == 7.0).all())
        assert bool((self.work[:GUARD] == 77).all()) and bool((self.work[GUARD + self.need:] == 77).all())
        same = zip((t.view(torch.uint8) for t in self.cache._kept + (self.q, self.cu, self.cuts, self.seqs)), (t.view(torch.uint8) for t in self.kept))
        assert all(torch.equal(a, b) for a, b in same)
        return inner.view(self.q.shape)


# prompts, forks of each, tokens of a fork's own, query tokens of each; the waits that there are
CASES = [([3000] * 60, 16, 600, 1, FEW),                       # 32 rows of a prefix and 2 of an item: few rows in both passes
         ([9000] * 8, 40, 300, 1, FEW + MANY),                 # 80 rows of a prefix: one tile of 128
         ([9000, 3000] * 4, 20, 700, 10, MANY),                # tiles of 256, and of 128 for what is an item's own
         ([9000] * 6, 10, 900, 150, MANY)]                     # tiles of 256 in both
PAIRS = [(case, code) for case in range(len(CASES)) for code in CASES[case][4]]


@pytest.mark.gpu
@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("case,code", PAIRS)
def test_expiry(case, code, asym):
    c = Call(*CASES[case][:4], asym)
    right = c.run()
    if code in (61, 71):
        check(c.cache, c.q, c.seqs.tolist(), c.cu.tolist(), c.cuts.tolist())
    assert c.plan.device_status() == 0
    seen = []
    for segment in range(4):
        c.run(code, segment)
        seen.append(c.plan.device_status())
        assert seen[-1] in (0, code)                           # 0: no block makes such a wait there
        assert torch.equal(c.run(), right)                     # the next call is as always
    assert code in seen
    c.plan.close()
