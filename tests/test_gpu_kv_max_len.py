"""max_len of the KV attention chooses how the work is split and nothing else."""
import pytest
import torch

import kv_norms
from kv_util import DEV, filled
from paper_2504_13989_b200 import KVCache, Plan
from paper_2504_13989_b200 import build as gbs_build

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("counts", [[1, 1, 1, 1], [2, 3, 1, 2], [60, 40, 7, 200]])
def test_sequences_that_are_longer(counts, asym):
    gbs_build.build()
    lengths = [5000, 40, 511, 700]
    with Plan(96, 128, 1, 4, 128, 0.9, asymmetric=asym) as plan:
        cache = filled(plan, lengths, 2, 16, seed=3)
        gen = torch.Generator(device=DEV)
        gen.manual_seed(1)
        q = torch.randn((sum(counts), 8, 96), generator=gen, device=DEV).to(torch.bfloat16)
        cu = torch.tensor([0] + counts, device=DEV).cumsum(0).to(torch.int32)
        for max_len in (1, 39, 512, 513, 4999, 5000, 2 ** 31 - 1):
            for window in (0, 100):
                got = cache.attention(q, None, cu, max(counts), max_len=max_len, window=window)
                kv_norms.check(cache, got, q, range(4), counts, window=window)


def test_a_captured_step_that_outgrows_it():
    """Every replay adds a token; the newest one is seen however many there are."""
    gbs_build.build()
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = KVCache.create(plan, 40, 2, 16, 2, 20, DEV)
        gen = torch.Generator(device=DEV)
        gen.manual_seed(2)
        cache.extend(None, torch.tensor([30, 60], dtype=torch.int32, device=DEV))
        k, v, q = (torch.randn((90, h, 128), generator=gen, device=DEV).to(torch.bfloat16) for h in (2, 2, 4))
        cache.append(k, v, None, torch.tensor([0, 30, 90], dtype=torch.int32, device=DEV))
        k, v, q = k[:2].clone(), v[:2].clone(), q[:2].clone()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            status = cache.extend()
            cache.append(k, v, status=status)
            got = cache.attention(q, max_len=64)
        for step in range(40):
            for t in (k, v, q):
                t.copy_(torch.randn(t.shape, generator=gen, device=DEV))
            g.replay()
            kv_norms.check(cache, got, q, range(2), [1, 1])
        assert cache.lengths.tolist() == [70, 100]
