"""gbs_kv_attention_mass for many query rows whose scores are large."""
import pytest
import torch

from kv_util import DEV, filled
from paper_2504_13989_b200 import Plan
from paper_2504_13989_b200 import build as gbs_build
from test_gpu_kv_mass import check, ints, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    gbs_build.build()


@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("scale", [3.0, -3.0, 1e20])
def test_large_scores(scale, asym):
    """Scores of some hundreds within the bound of the other tests; of 10^21, where fp32 has no units, weights are finite all the same."""
    with Plan(128, 128, 1, 4, 128, 0.9, asymmetric=asym) as plan:
        cache = filled(plan, [2000, 129], 2, 64, seed=2)
        q = rows(90, 8, 128, 1, 2.0)
        if abs(scale) < 1e3:
            check(cache, q, [0, 1], [0, 60, 90], scale=scale, decay=0.5)
            check(cache, q, [0, 1], [0, 60, 90], scale=scale, decay=0.0, window=300)
        else:
            mass = cache.attention_mass(q, torch.zeros((2, 2, 2000), device=DEV), None, ints([0, 60, 90]), 60, scale=scale)
            assert bool(mass.isfinite().all()) and bool((mass >= 0).all())
