"""Which form a windowed-attention call takes, and what its plan is (csrc/attend_plan.h), without a GPU."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2604_09244_b200 import mvla

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FMA, TILE, TOKEN = 0, 1, 2
SHIM = r"""
#include "serve_checks.h"
using namespace mvla;
extern "C" int32_t plan(int dtype, int H, int G, int d, int32_t n, const mvla_seq* s, int mass, int32_t window, int32_t sinks, int64_t* out)
{
    const ServeShape v = {dtype, dtype == 1 ? 1 : 0, H, G, d, 64, 148, size_t(dtype == 1 ? 4 : dtype == 0 ? 2 : 1), size_t(dtype == 1 ? 4 : 2)};
    const AttendPlan p = plan_attend(v, n, s, true, window, sinks, mass != 0);
    int64_t blocks = 0, most = 0;
    for (int b = 0; b < n; ++b) {
        const int32_t parts = parts_of(p, s[b], true, window, sinks);
        blocks += parts;
        most = parts > most ? parts : most;
    }
    out[0] = p.splits; out[1] = p.blocks; out[2] = p.bytes; out[3] = blocks; out[4] = most;
    return p.form;
}
"""


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    src, lib = str(d / "shim.cpp"), str(d / "shim.so")
    open(src, "w").write(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_2604_09244_b200", "csrc"), src, "-o", lib], check=True)
    return C.CDLL(lib)


def form(shim, dtype, heads, lens, n_q=1, mass=False, window=mvla.WINDOW_ALL, sinks=0):
    at, seqs = 0, []
    for b, n in enumerate(lens):
        seqs.append(mvla.Seq(q_row=b * n_q, n_q=n_q, kv_row=at, n_kv=n))
        at += n
    out = (C.c_int64 * 5)()
    f = shim.plan(dtype, *heads, len(seqs), mvla.c_seqs(seqs), mass, window, sinks, out)
    assert 1 <= out[0] and out[2] >= 0
    if f == TOKEN:
        assert out[1] == out[3] and out[0] == max(1, out[4]) and out[0] <= 256
    return f


BF16, FP32, FP8 = mvla.DTYPE_BF16, mvla.DTYPE_FP32, mvla.DTYPE_FP8_E4M3
GROUPED, EACH = (32, 8, 128), (32, 32, 128)


@pytest.mark.parametrize("want,dtype,heads,lens,kw", [
    # short calls of a few rows: measured 8.5 us by tokens, 12.8 by tiles (800 rows); 12.4 and 14.2 (4000)
    (TOKEN, BF16, GROUPED, [800], {}), (TOKEN, BF16, EACH, [800], {}), (TOKEN, BF16, GROUPED, [4000], {}), (TOKEN, BF16, GROUPED, [1], {}),
    (TOKEN, BF16, GROUPED, [2000, 2000], {}), (TOKEN, BF16, GROUPED, [60000], dict(window=500, sinks=4)),
    # long ones, and more than eight rows to a key head
    (TILE, BF16, GROUPED, [16000], {}), (TILE, BF16, EACH, [16000], {}), (TILE, BF16, GROUPED, [750] * 32, {}), (TILE, BF16, GROUPED, [200], dict(n_q=3)),
    (TILE, BF16, GROUPED, [30000], dict(n_q=4)), (TILE, BF16, GROUPED, [200], dict(n_q=5)), (TILE, BF16, (16, 16, 64), [300], dict(n_q=40)),
    # weights, heads of 64, unlike lengths, e4m3
    (TOKEN, BF16, GROUPED, [60000], dict(mass=True)), (TOKEN, BF16, (16, 16, 64), [60000], {}), (TOKEN, BF16, GROUPED, [500, 20000, 900, 300], {}),
    (TOKEN, FP8, GROUPED, [60000], {}), (TILE, FP8, GROUPED, [60000], dict(n_q=5)), (FMA, FP32, GROUPED, [60000], {}), (FMA, FP32, GROUPED, [60], dict(n_q=60)),
])
def test_form_of_a_call(shim, want, dtype, heads, lens, kw):
    assert form(shim, dtype, heads, lens, **kw) == want
