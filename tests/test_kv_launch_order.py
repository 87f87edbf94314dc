"""Kernels of the paged KV cache start while the launch before them ends, and touch no memory of the caller's before they have waited for it.

griddepcontrol.wait makes what earlier launches wrote visible to the grid that waits, and to nobody else: that the launch before has itself waited is not enough."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2504_13989_b200", "csrc")
FILES = sorted(f for pat in ("gbs_kv_*.cu", "gbs_kv_*.cuh", "gbs_tc_kv*.cu") for f in glob.glob(os.path.join(CSRC, pat)))
# what reads the call's arrays
READS = re.compile(r"\b(kv_length|kv_sequence|kv_item|kv_item_of|kv_entry|kv_share|kv_page|kv_start_of|weight|atomic\w+)\(|\b[APE]\.(c\.)?"
                   r"(mass|base|lengths|page_table|refs|status|kept|seqs|cu|groups|joins|parts|fresh|weights|q|pages)\[")


def kernels():
    for path in FILES:
        text = re.sub(r"//[^\n]*", "", open(path).read())
        for m in re.finditer(r"__global__[^;{]*?\b(k_\w+)\(", text):
            start = text.index("\n{", m.end())
            yield os.path.basename(path), m.group(1), text[start:text.index("\n}", start)]


def test_the_files_have_kernels():
    found = {(f, k) for f, k, _ in kernels()}
    assert len(FILES) >= 9 and len(found) >= 20 and ("gbs_kv_evict.cu", "k_kv_select") in found and ("gbs_tc_kvattn.cu", "k_tc_kvattn") in found


@pytest.mark.parametrize("file,kernel,body", [pytest.param(*k, id="%s-%d" % (k[1], i)) for i, k in enumerate(kernels())])
def test_a_kernel_waits_before_it_reads(file, kernel, body):
    assert body.count("kv_wait_before();") == 1, (file, kernel)
    assert not READS.search(body[:body.index("kv_wait_before();")]), (file, kernel)
