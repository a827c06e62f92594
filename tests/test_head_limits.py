"""Limits of the rules' counts, without a GPU: refused before any CUDA call."""
import os
import re

import pytest

from paper_2608_02438_gb300 import binding as X
from paper_2608_02438_gb300 import build as BLD


@pytest.fixture(scope="module")
def lib():
    BLD.build()
    return X.load()


def test_a_history_that_a_count_cannot_hold(lib):
    """A count has 30 bits: 2^30 times the same token would read as a token of the block."""
    g = X.XpressLogitsArgs(n_seq=1, rows=2, V=1000, dtype=X.XPRESS_BF16, logits=4096, ld=1000, out=8192, ldo=1000,
                           repetition=4096, history=4096, n_history=1 << 30, history_offsets=4096)
    assert lib.xpress_process_logits(g, None, 0, None) == X.XPRESS_ERR_UNSUPPORTED


def test_counts_are_declared_as_they_are_read():
    """The dynamic shared memory of csrc/logits.cu is read and cleared 16 bytes at a time: it
    has to be declared on 16 bytes, whatever lies before it."""
    with open(os.path.join(BLD.CSRC, "logits.cu")) as f:
        src = f.read()
    assert re.search(r"reinterpret_cast<(const )?uint4 \*>\(cnt\b", src)
    assert re.findall(r"extern __shared__ (.*?)uint32_t cnt\[\]", src) == ["__align__(16) "]
