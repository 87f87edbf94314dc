"""extend and fork with as many items as a call may have, and from several host threads at once."""
import ctypes
import random
import threading

import pytest
import torch

from kv_util import DEV, Model
from paper_2504_13989_b200 import KVCache, Plan, binding
from paper_2504_13989_b200 import build as gbs_build

pytestmark = pytest.mark.gpu
MOST = binding.GBS_KV_MAX_ITEMS


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def test_the_most_items():
    gbs_build.build()
    rng = random.Random(1)
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        cache = KVCache.create(plan, 16000, 1, 16, MOST, 4, DEV)
        model = Model(16000, 16, MOST, 4)
        assert cache.extend().tolist() == model.extend(list(range(MOST)), [1] * MOST)
        model.check(cache)
        seqs = [rng.randrange(-2, MOST + 2) for _ in range(MOST)]
        counts = [rng.randrange(-1, 40) for _ in range(MOST)]
        assert cache.extend(ints(seqs), ints(counts)).tolist() == model.extend(seqs, counts)
        model.check(cache)
        gone = rng.sample(range(MOST), MOST // 2)
        cache.free(ints(gone))
        model.free(gone)
        src, dst = [rng.randrange(MOST) for _ in range(MOST)], [rng.choice(gone) for _ in range(MOST)]
        assert cache.fork(ints(src), ints(dst)).tolist() == model.fork(src, dst)
        model.check(cache)
        everything = list(range(MOST))
        cache.free(ints(everything))
        model.free(everything)
        model.check(cache)
        assert not cache.refs.any()


def test_calls_of_different_sizes_from_several_threads():
    """Straight into the library, which no lock guards: every call is made, each thread's on a pool and a stream of its own."""
    gbs_build.build()
    lib = binding.lib()
    with Plan(128, 128, 1, 4, 128, 0.9) as plan:
        sizes, failed, pools = (MOST, 3000, 5000), [], []
        for n in sizes:
            cache = KVCache.create(plan, 2 * n, 1, 16, n, 40, DEV)
            pools.append((cache, torch.empty(n, dtype=torch.int32, device=DEV), torch.cuda.Stream(), n))
        torch.cuda.synchronize()

        def work(cache, status, stream, n):
            for _ in range(300):
                rc = lib.gbs_kv_extend(plan.handle, ctypes.byref(cache._c), None, None, n, status.data_ptr(), stream.cuda_stream)
                if rc != 0:
                    failed.append((n, rc))
        threads = [threading.Thread(target=work, args=p) for p in pools]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        torch.cuda.synchronize()
        assert not failed
        for cache, status, _, n in pools:                      # two pages a sequence: 32 tokens, and no room for the 33rd of any
            assert cache.lengths.tolist() == [32] * n and bool((status == binding.GBS_KV_NO_PAGES).all())
