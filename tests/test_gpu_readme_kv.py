"""The readme's examples of the KV cache: they run as they stand, and the one that shares a prefix has sizes by which it is shared."""
import ctypes
import os
import re

import pytest
import torch

from paper_2504_13989_b200 import binding
from paper_2504_13989_b200 import build as gbs_build

README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


def blocks():
    found = [b for b in re.findall(r"```python\n(.*?)```", open(README).read(), re.S) if "cache." in b]
    assert len(found) == 2
    return found


def shared_bytes(handle, cache, items, max_prefix):
    """Workspace of a step of so many forks, 32 query heads."""
    need = ctypes.c_int64(0)
    assert binding.lib().gbs_kv_shared_attention_workspace(handle, ctypes.byref(cache), items, items, 1, 1, max_prefix, 32, ctypes.byref(need)) == 0
    return need.value


@pytest.mark.gpu
def test_they_run():
    gbs_build.build()
    names = {"torch": torch}                                   # the first block of the file imports it
    torch.manual_seed(1)
    for b in blocks():
        exec(b, names)                                         # noqa: S102
    torch.cuda.synchronize()
    cache, forks = names["cache"], names["forks"]
    n, prefix = len(forks), int(re.search(r"max_prefix=(\d+)", blocks()[1]).group(1))
    assert names["status"].eq(0).all() and cache.lengths[forks.long()].eq(256).all() and int(cache.lengths[7]) == 6000
    assert names["out"].isfinite().all() and names["kept"].ge(0).all() and names["mass"].isfinite().all()
    # rows of 528 bytes wait for their own parts where a prefix is shared
    assert shared_bytes(names["plan"].handle, cache._c, n, prefix) - shared_bytes(names["plan"].handle, cache._c, n, 1) > n * 32 * 500
    # 32 tokens of 32 heads weighed the document
    assert abs(float(names["mass"][7].double().sum()) - 32 * 32) < 0.1
    assert names["plan"].device_status() == 0
