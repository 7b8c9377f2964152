"""Kernels by tiles whose CTAs join their sums inside clusters hold no tensor memory while they wait for one another.

A cluster's CTAs are placed together by registers, threads and shared memory, but not by tensor memory, whose allocation waits.  Launches of two shapes on two streams can
fill a multiprocessor with CTAs that ask for more than its 512 columns (heads of 64: 78 KB and 256 columns beside 114 KB and 512).  CTA A of one launch then holds columns on
multiprocessor X and B of the other on Y, A's peer waits on Y for B's columns and B's peer on X for A's: none of them ends.  Shown by reading: a run of it would hang."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_09244_b200", "csrc")


@pytest.mark.parametrize("name", ["attend_tile.cu", "page_tile.cu"])
def test_columns_are_given_back_before_the_cluster_meets(name):
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    kernels = [k for k in re.split(r"__global__", text)[1:] if "join_cluster<" in k]
    assert kernels
    for k in kernels:
        assert k.count("tmem_dealloc(") == 1 and k.index("tmem_alloc(") < k.index("tmem_dealloc(") < k.index("cluster_arrive_release(") < k.index("join_cluster<")
