"""Threads of the kernels that copy rows into pages and out of them (csrc/page_plan.h: row_slot): every lane of every head has its thread, and no thread, the surplus
ones among them, has a head that the pool has not.  Host arithmetic, without a GPU."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SHIM = r"""
#include "page_plan.h"
using namespace mvla;
extern "C" int slots(int lanes, int kv_heads, int keys, int values, int32_t* out)
{
    const int all = ((keys ? kv_heads : 0) + (values ? kv_heads : 0)) * lanes, columns = (all + kRowThreads - 1) / kRowThreads;
    for (int c = 0; c < columns; ++c)
        for (int t = 0; t < kRowThreads; ++t) {
            const RowSlot s = row_slot(t, c, lanes, kv_heads, keys, values);
            const int32_t one[] = {s.values, s.on, s.head, s.lane, s.first, s.step};
            for (int i = 0; i < 6; ++i) *out++ = one[i];
        }
    return columns * kRowThreads;
}
"""


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    d = tmp_path_factory.mktemp("shim")
    src, lib = str(d / "shim.cpp"), str(d / "shim.so")
    open(src, "w").write(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_2604_09244_b200", "csrc"), src, "-o", lib], check=True)
    return C.CDLL(lib)


@pytest.mark.parametrize("keys,values", [(1, 1), (1, 0), (0, 1)])
@pytest.mark.parametrize("lanes", [4, 8, 16])
def test_every_lane_has_a_thread_and_no_thread_a_head_outside_the_pool(shim, lanes, keys, values):
    out = np.zeros((1 << 16, 6), dtype=np.int32)
    for kv_heads in list(range(1, 130)) + [255, 256, 257]:
        n = shim.slots(lanes, kv_heads, keys, values, out.ctypes.data_as(C.POINTER(C.c_int32)))
        tensor, on, head, lane, first, step = out[:n].T
        # whether it copies or not: what it forms addresses of is there
        assert ((head >= 0) & (head < kv_heads)).all(), kv_heads
        assert ((tensor == 1) <= (values == 1)).all() and ((tensor == 0) <= (keys == 1)).all()
        assert ((lane >= 0) & (lane < lanes)).all() and (step == step[0]).all()
        # those that copy: each lane of each head of each tensor once in every one of the rows that go side by side
        on = on.astype(bool)
        assert ((first[on] >= 0) & (first[on] < step[0])).all()
        key = ((first[on].astype(np.int64) * 2 + tensor[on]) * kv_heads + head[on]) * lanes + lane[on]
        assert len(key) == len(np.unique(key)) == step[0] * (keys + values) * kv_heads * lanes
