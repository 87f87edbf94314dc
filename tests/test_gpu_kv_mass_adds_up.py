"""gbs_kv_attention_mass: a row's weights add up to 1, however large its scores are."""
import math

import pytest
import torch

import kv_util
from kv_util import DEV, filled
from paper_2504_13989_b200 import Plan
from paper_2504_13989_b200 import build as gbs_build
from test_gpu_kv_mass import cu_of, ints, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    gbs_build.build()


@pytest.mark.parametrize("count", [10, 20, 300])             # 40, 80 and 1200 rows of a KV head: one tile, two, and a ring of them
@pytest.mark.parametrize("scale", [100.0, -100.0, 1.0])
def test_many_rows(count, scale):
    """The same query row again and again, so that what is off is off in the same direction.

    Relative, in units of 2^-24, S the largest score in units of log2: a score in the first pass may be rounded by its own size before m is taken from it, and so is the logarithm of a row's sum:
    2 x 0.69 S.  log2f: a unit in the last place of 16 .. 32, twice 16 x 0.69.  z - m is rounded by |z - m| <= 20 on average over a row's weight (11.6 for an even softmax over 3000, and m within 8 of
    the largest): 2 x 20 x 0.69 = 28.  ex2 on either side: 2 x 4.  The sum of a row: 48 additions of a thread and 5 within sixteen tokens, 4 parts, pieces of the blocks that share a segment (12 at
    most, with two factors each: 36).  A token's sum over a tile: 16, and 4 for the rest, which is compensated."""
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = filled(plan, [3000, 3000, 3000], 1, 32, seed=2)
        for seed in range(4):
            q = rows(3, 4, 128, seed)[:, :1].expand(3, 4, 128).repeat_interleave(count, 0).contiguous()
            mass = torch.full((3, 1, 3000), float("nan"), device=DEV)
            cache.attention_mass(q, mass, None, ints(cu_of([count] * 3)), count, decay=0.0, causal=False, scale=scale)
            off = (mass.double().sum((1, 2)) / (4 * count) - 1).abs()
            x = q[::count, 0].double() @ kv_util.h128() / 128 ** 0.5
            largest = torch.stack([(kv_util.rows_of(cache, i)[0][0] @ x[i]).abs().max() for i in range(3)]) * abs(scale) / math.log(2)
            assert bool((off <= (1.39 * largest + 22 + 28 + 8 + 53 + 4 + 36 + 20) * 2.0 ** -24).all()), (off / largest).tolist()


@pytest.mark.parametrize("count,width", [(1, 3000), (8, 3000), (8, (1 << 26) // (3 * 32) + 1)])     # scores kept from the first pass, and found again
@pytest.mark.parametrize("scale", [100.0, -100.0])
def test_few_rows(count, width, scale):
    """As above: 2 x 4 for ex2 (z - m is the same number on both sides); 24 additions of a thread for a row's sum, 8 within a warp, 4 parts, pieces of the blocks as above; 2; a token's sum
    over 8 rows at a time and then over four lanes: 10, and 4 for the rest."""
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = filled(plan, [3000, 3000, 3000], 1, 32, seed=2)
        for seed in range(4):
            q = rows(3, 4, 128, seed)[:, :1].expand(3, 4, 128).repeat_interleave(count, 0).contiguous()
            mass = torch.zeros((3, 1, width), device=DEV)
            cache.attention_mass(q, mass, None, ints(cu_of([count] * 3)), count, decay=0.0, causal=False, scale=scale)
            off = (mass[..., :3000].double().sum((1, 2)) / (4 * count) - 1).abs()
            assert bool((off <= 100 * 2.0 ** -24).all()), off.tolist()
