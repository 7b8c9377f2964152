"""Host side of the calls around the prune point (csrc/serve_checks.h): refusals and workspaces, without a GPU, through a small
library built from the header itself; and what the exported calls answer without a context."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2604_09244_b200 import mvla

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SHIM = r"""
#include "serve_checks.h"
using namespace mvla;
static ServeShape shape(int dtype, int H, int G, int d)
{
    return {dtype, dtype == 1 ? 1 : 0, H, G, d, 4, 148, size_t(dtype == 1 ? 4 : dtype == 0 ? 2 : 1), size_t(dtype == 1 ? 4 : 2)};
}
extern "C" int32_t rope(int dtype, int H, int G, int d, const mvla_qk_rope* r) { return check_rope(shape(dtype, H, G, d), r); }
extern "C" int32_t attention(int dtype, int H, int G, int d, int32_t n, const mvla_seq* s, const mvla_attention* a, int64_t* bytes)
{
    const ServeShape v = shape(dtype, H, G, d);
    int32_t rc = check_attention(v, n, s, a);
    if (rc != MVLA_OK) return rc;
    const AttendPlan p = plan_of(v, n, s, a);
    *bytes = p.bytes;
    return p.total_q ? check_attention_memory(v, n, a, p) : MVLA_OK;
}
extern "C" int32_t eviction(int dtype, int H, int G, int d, int32_t n, const mvla_seq* s, const mvla_eviction* a, int64_t* bytes)
{
    const ServeShape v = shape(dtype, H, G, d);
    int32_t rc = check_eviction(v, n, s, a);
    if (rc != MVLA_OK) return rc;
    const EvictPlan p = plan_evict(n, s);
    *bytes = p.bytes;
    return check_eviction_memory(v, n, a, p);
}
"""
BF16, FP32, FP8 = mvla.DTYPE_BF16, mvla.DTYPE_FP32, mvla.DTYPE_FP8_E4M3
OK, BAD, UNSUP, CAP = mvla.OK, mvla.ERR_INVALID_ARG, mvla.ERR_UNSUPPORTED, mvla.ERR_CAPACITY
MB = 1 << 20


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    d = tmp_path_factory.mktemp("shim")
    src, lib = str(d / "shim.cpp"), str(d / "shim.so")
    open(src, "w").write(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_2604_09244_b200", "csrc"), src, "-o", lib], check=True)
    return C.CDLL(lib)


def test_struct_sizes():
    assert C.sizeof(mvla.CSeq) == 2 * 8 + 4 * 4
    assert C.sizeof(mvla.CQkRope) == 11 * 8 + 2 * 4 + 8 + 5 * 8
    assert C.sizeof(mvla.CAttention) == 8 * 8 + 2 * 4 + 6 * 8
    assert C.sizeof(mvla.CEviction) == 10 * 8 + 2 * 4 + 2 * 8


def test_calls_without_a_context():
    lib = mvla.load_library()
    n = C.c_int64()
    assert lib.mvla_qk_norm_rope(None, C.byref(mvla.CQkRope()), None) == BAD
    assert lib.mvla_window_attention(None, 1, None, C.byref(mvla.CAttention()), None) == BAD
    assert lib.mvla_window_attention_workspace(None, 1, None, C.byref(mvla.CAttention()), C.byref(n)) == BAD
    assert lib.mvla_cache_evict(None, 1, None, C.byref(mvla.CEviction()), None) == BAD
    assert lib.mvla_cache_evict_workspace(None, 1, None, C.byref(mvla.CEviction()), C.byref(n)) == BAD


def rope_args(**kw):
    a = dict(q=1 * MB, k=2 * MB, v=3 * MB, n_rows=10, q_stride=512, k_stride=256, v_stride=256, pos=4 * MB, inv_freq=5 * MB, rot_dim=64, flags=1,
             eps=1e-6, q_out=6 * MB, k_out=7 * MB, v_out=8 * MB, kv_rows=10)
    a.update(kw)
    return mvla.CQkRope(**a)


@pytest.mark.parametrize("want,kw", [
    (OK, {}), (OK, dict(n_rows=0, pos=None)), (OK, dict(q=None, q_out=None)), (OK, dict(rot_dim=0, pos=None, inv_freq=None)),
    (OK, dict(q_out=1 * MB, k_out=2 * MB)), (OK, dict(out_rows=9 * MB, kv_rows=3)), (OK, dict(q_weight=9 * MB)), (OK, dict(n_rows=1, kv_rows=1, q_stride=0)),
    (BAD, dict(n_rows=-1)), (BAD, dict(pos=None)), (BAD, dict(inv_freq=None)), (BAD, dict(rot_dim=80)), (UNSUP, dict(rot_dim=40)),
    (BAD, dict(flags=4)), (BAD, dict(flags=0, q_weight=9 * MB)), (BAD, dict(eps=-1.0)), (BAD, dict(eps=float("nan"))), (BAD, dict(q_out=None)),
    (BAD, dict(k=None)), (BAD, dict(q=1 * MB + 8)), (BAD, dict(q_stride=511)), (BAD, dict(q_stride=516)), (BAD, dict(kv_rows=9)),
    (BAD, dict(q_out=1 * MB + 1024)), (BAD, dict(q_out=1 * MB, q_stride=640)), (BAD, dict(k_out=2 * MB, out_rows=9 * MB)), (BAD, dict(k_out=1 * MB)),
    (BAD, dict(v_out=7 * MB)), (BAD, dict(pos=4 * MB + 2)), (BAD, dict(kv_rows=1 << 60)), (BAD, dict(q_stride=1 << 60)), (BAD, dict(q_out=4 * MB)),
    (BAD, dict(k_out=5 * MB)), (BAD, dict(v_out=9 * MB, out_rows=9 * MB)), (BAD, dict(q_out=9 * MB, k_weight=9 * MB)),
])
def test_rope_refusals(shim, want, kw):
    assert shim.rope(BF16, 8, 4, 64, C.byref(rope_args(**kw))) == want


def test_rope_of_e4m3_cannot_be_in_place(shim):
    assert shim.rope(FP8, 8, 4, 64, C.byref(rope_args())) == OK
    assert shim.rope(FP8, 8, 4, 64, C.byref(rope_args(q_out=1 * MB))) == BAD


def attention_call(shim, seqs, dtype=BF16, heads=(8, 4, 64), **kw):
    a = dict(q=1 * MB, k=16 * MB, v=32 * MB, q_rows=100, kv_rows=1000, window=mvla.WINDOW_ALL, n_sink=0, scale=0.0, out=2 * MB, workspace=64 * MB,
             workspace_bytes=1 << 40)
    a.update(kw)
    n = C.c_int64(-1)
    c = mvla.c_seqs([mvla.Seq(**s) for s in seqs])
    return shim.attention(dtype, *heads, len(seqs), c, C.byref(mvla.CAttention(**a)), C.byref(n)), n.value


ONE = [dict(n_q=3, n_kv=40)]


@pytest.mark.parametrize("want,seqs,kw", [
    (OK, ONE, {}), (OK, [dict(n_q=0, n_kv=0)] * 4, {}), (OK, [dict(n_q=2, n_kv=0)], dict(k=None, v=None)),
    (OK, [dict(n_q=1, n_kv=40), dict(q_row=1, n_q=1, n_kv=40)], {}),
    (OK, [dict(q_row=50, n_q=50, kv_row=500, n_kv=500), dict(q_row=0, n_q=50, kv_row=0, n_kv=500)], dict(mass=3 * MB)),
    (CAP, ONE * 5, {}), (BAD, [], {}), (BAD, [dict(n_q=-1, n_kv=40)], {}), (BAD, [dict(n_q=1, n_kv=-1)], {}), (BAD, [dict(q_row=98, n_q=3, n_kv=1)], {}),
    (BAD, [dict(q_row=1 << 62, n_q=3, n_kv=1)], {}), (BAD, [dict(kv_row=1 << 62, n_q=3, n_kv=1)], {}), (BAD, [dict(kv_row=990, n_q=3, n_kv=11)], {}),
    (BAD, [dict(n_q=2, n_kv=4), dict(q_row=1, n_q=2, kv_row=9, n_kv=4)], {}),
    (BAD, [dict(n_q=2, n_kv=4), dict(q_row=2, n_q=2, kv_row=3, n_kv=4)], dict(mass=3 * MB)),
    (BAD, [dict(q_row=9, n_q=2, kv_row=3, n_kv=4), dict(q_row=2, n_q=2, kv_row=6, n_kv=4)], dict(mass=3 * MB)),
    (BAD, ONE, dict(window=0)), (BAD, ONE, dict(n_sink=-1)), (BAD, ONE, dict(scale=-1.0)), (BAD, ONE, dict(scale=float("inf"))),
    (BAD, ONE, dict(kv_pos=3 * MB)), (OK, ONE, dict(kv_pos=3 * MB, q_pos=4 * MB)), (BAD, ONE, dict(kv_pos=3 * MB + 2, q_pos=4 * MB)),
    (BAD, ONE, dict(q=None)), (BAD, ONE, dict(k=None)), (BAD, ONE, dict(out=None)), (BAD, ONE, dict(out=1 * MB)), (BAD, ONE, dict(out=16 * MB + 1024)),
    (BAD, ONE, dict(q=1 * MB + 2)), (BAD, ONE, dict(lse=2 * MB)), (BAD, ONE, dict(mass=2 * MB)), (BAD, ONE, dict(mass=16 * MB)),
    (BAD, ONE, dict(mass=3 * MB, workspace=None)), (BAD, ONE, dict(mass=3 * MB, workspace_bytes=8)), (BAD, ONE, dict(mass=3 * MB, workspace=64 * MB + 16)),
    (BAD, ONE, dict(mass=3 * MB, workspace=16 * MB)), (BAD, ONE, dict(q_rows=-1)), (BAD, ONE, dict(kv_rows=1 << 60)),
])
def test_attention_refusals(shim, want, seqs, kw):
    assert attention_call(shim, seqs, **kw)[0] == want


def eviction_call(shim, seqs, **kw):
    a = dict(k=16 * MB, v=32 * MB, kv_rows=1000, pos=1 * MB, mass=2 * MB, pos_out=1 * MB, mass_out=2 * MB, n_sink=2, n_recent=3, workspace=64 * MB,
             workspace_bytes=1 << 40)
    a.update(kw)
    n = C.c_int64(-1)
    c = mvla.c_seqs([mvla.Seq(**s) for s in seqs])
    return shim.eviction(BF16, 8, 4, 64, len(seqs), c, C.byref(mvla.CEviction(**a)), C.byref(n))


EV = [dict(n_kv=40, budget=20)]


@pytest.mark.parametrize("want,seqs,kw", [
    (OK, EV, {}), (OK, EV, dict(pos_out=3 * MB, mass_out=4 * MB, kept_idx=5 * MB, kv_len=6 * MB, kv_len_out=6 * MB)),
    (OK, [dict(n_kv=0, budget=5)], {}), (OK, [dict(n_kv=40, budget=2000)], {}), (OK, [dict(kv_row=40, n_kv=40, budget=9), dict(n_kv=40, budget=9)], {}),
    (CAP, EV * 5, {}), (BAD, [dict(n_kv=40, budget=4)], {}), (BAD, [dict(n_kv=40, budget=-1)], dict(n_sink=0, n_recent=0)),
    (BAD, EV, dict(n_sink=-1)), (BAD, EV, dict(n_sink=0x7FFFFFFF, n_recent=0x7FFFFFFF)), (BAD, [dict(n_kv=40, budget=9), dict(kv_row=39, n_kv=4, budget=9)], {}),
    (BAD, [dict(kv_row=990, n_kv=40, budget=9)], {}), (BAD, EV, dict(k=None)), (BAD, EV, dict(v=16 * MB)), (BAD, EV, dict(v=16 * MB + 4096)),
    (BAD, EV, dict(pos=None)), (BAD, EV, dict(mass_out=None)), (BAD, EV, dict(pos_out=1 * MB + 4)), (BAD, EV, dict(pos_out=2 * MB)),
    (BAD, EV, dict(kept_idx=1 * MB)), (BAD, EV, dict(workspace=None)), (BAD, EV, dict(workspace_bytes=100)), (BAD, EV, dict(workspace=16 * MB)),
    (BAD, EV, dict(kv_len_out=1 * MB)), (BAD, EV, dict(k=16 * MB + 8)),
])
def test_eviction_refusals(shim, want, seqs, kw):
    assert eviction_call(shim, seqs, **kw) == want
