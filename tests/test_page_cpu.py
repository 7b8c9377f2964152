"""Host side of the calls on a cache in pages (csrc/page_checks.h): refusals and workspaces, without a GPU, through a small library
built from the header itself; what the exported calls answer without a context; and the reference's own rounding."""
import ctypes as C
import os
import subprocess

import pytest
import torch

import page_util as P
from paper_2604_09244_b200 import mvla

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SHIM = r"""
#include "page_checks.h"
using namespace mvla;
static ServeShape shape(int dtype, int H, int G, int d)
{
    return {dtype, dtype == 1 ? 1 : 0, H, G, d, 4, 148, size_t(dtype == 1 ? 4 : dtype == 0 ? 2 : 1), size_t(dtype == 1 ? 4 : 2)};
}
extern "C" int32_t rows(int dtype, int H, int G, int d, int32_t n, const mvla_seq* s, const mvla_page_rows* a, int write)
{
    return check_page_rows(shape(dtype, H, G, d), n, s, a, write != 0);
}
extern "C" int32_t attention(int dtype, int H, int G, int d, int32_t n, const mvla_seq* s, const mvla_paged_attention* a, int64_t* bytes)
{
    const ServeShape v = shape(dtype, H, G, d);
    const int32_t rc = check_page_attention(v, n, s, a);
    if (rc != MVLA_OK) return rc;
    const PageAttendPlan p = plan_page_attention(v, n, s, a);
    *bytes = p.bytes;
    return p.attend.total_q ? check_page_attention_memory(v, n, a, p) : MVLA_OK;
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
    assert C.sizeof(mvla.CPages) == 5 * 8 + 2 * 4
    assert C.sizeof(mvla.CPageRows) == 48 + 8 * 8
    assert C.sizeof(mvla.CPagedAttention) == 48 + 5 * 8 + 2 * 4 + 5 * 8


def test_calls_without_a_context():
    lib = mvla.load_library()
    n = C.c_int64()
    assert lib.mvla_page_write(None, 1, None, C.byref(mvla.CPageRows()), None) == BAD
    assert lib.mvla_page_read(None, 1, None, C.byref(mvla.CPageRows()), None) == BAD
    assert lib.mvla_page_attention(None, 1, None, C.byref(mvla.CPagedAttention()), None) == BAD
    assert lib.mvla_page_attention_workspace(None, 1, None, C.byref(mvla.CPagedAttention()), C.byref(n)) == BAD


def pages(**kw):
    """100 pages of 64 rows of 4 heads of 64: 3.2 MB of bf16 each, 1.6 MB of e4m3, 25600 scale bytes."""
    a = dict(k=16 * MB, v=32 * MB, n_pages=100, page_rows=64, kind=mvla.PAGE_ROWS)
    if kw.get("kind"):
        a.update(k_scale=48 * MB, v_scale=49 * MB)
    a.update(kw)
    return mvla.CPages(**a)


def rows_call(shim, seqs, pool, write, dtype=BF16, **kw):
    a = dict(pages=pool, table=1 * MB, table_stride=8, k=2 * MB, v=3 * MB, rows=100, k_stride=256, v_stride=256)
    a.update(kw)
    return shim.rows(dtype, 8, 4, 64, len(seqs), mvla.c_seqs([mvla.Seq(**s) for s in seqs]), C.byref(mvla.CPageRows(**a)), int(write))


ONE = [dict(n_q=3, n_kv=40)]
MANY = [dict(n_q=400, n_kv=500)]           # unpacked first: a call that needs a workspace
KINDS = dict(e4m3=dict(kind=mvla.PAGE_E4M3), e2m1=dict(kind=mvla.PAGE_E2M1))


@pytest.mark.parametrize("write", [True, False])
@pytest.mark.parametrize("want,seqs,pool,kw", [
    (OK, ONE, {}, {}), (OK, ONE, KINDS["e4m3"], {}), (OK, ONE, KINDS["e2m1"], {}), (OK, ONE, {}, dict(k=None)), (OK, ONE, {}, dict(k=None, v=None)),
    (OK, [dict(n_q=0, n_kv=0)] * 4, dict(k=None, v=None), dict(table=None)), (OK, [dict(n_q=512, n_kv=512)], {}, dict(rows=512)),
    (OK, ONE, {}, dict(k=2 * MB, v=2 * MB + 512, k_stride=512, v_stride=512)), (OK, [dict(n_q=5, n_kv=0)], {}, dict(table=None, table_stride=0)),
    (OK, ONE, dict(n_pages=0, k=None, v=None), {}), (OK, [dict(n_q=100, n_kv=40)], {}, {}),
    (CAP, ONE * 5, {}, {}), (BAD, [], {}, {}), (BAD, [dict(n_q=-1, n_kv=40)], {}, {}), (BAD, [dict(n_q=1, n_kv=-1)], {}, {}),
    (BAD, [dict(q_row=98, n_q=3, n_kv=40)], {}, {}), (BAD, [dict(q_row=1 << 62, n_q=3, n_kv=4)], {}, {}), (BAD, [dict(n_q=1, n_kv=513)], {}, {}),
    (BAD, ONE, dict(kind=3, k_scale=48 * MB, v_scale=49 * MB), {}), (BAD, ONE, dict(kind=-1), {}), (BAD, ONE, dict(n_pages=-1), {}),
    (UNSUP, ONE, dict(page_rows=8), {}), (UNSUP, ONE, dict(page_rows=48), {}), (UNSUP, ONE, dict(page_rows=512), {}), (UNSUP, ONE, dict(n_pages=1 << 30), {}),
    (UNSUP, ONE, dict(n_pages=1 << 40), {}),
    (BAD, ONE, dict(k=None), {}), (BAD, ONE, dict(v=None), {}), (BAD, ONE, dict(k_scale=48 * MB), {}), (BAD, ONE, dict(k=16 * MB + 8), {}),
    (BAD, ONE, dict(kind=mvla.PAGE_E4M3, k_scale=None), {}), (BAD, ONE, dict(kind=mvla.PAGE_E2M1, v_scale=49 * MB + 4), {}),
    (BAD, ONE, dict(v=16 * MB + 3 * MB), {}), (OK, ONE, dict(kind=mvla.PAGE_E4M3, v=16 * MB + 3 * MB), {}), (BAD, ONE, dict(kind=mvla.PAGE_E4M3, v_scale=48 * MB + 16), {}),
    (BAD, ONE, dict(kind=mvla.PAGE_E4M3, k_scale=16 * MB), {}),
    (BAD, ONE, {}, dict(table=None)), (BAD, ONE, {}, dict(table=1 * MB + 2)), (BAD, ONE, {}, dict(table_stride=-1)), (BAD, ONE, {}, dict(kv_len=1 * MB + 1)),
    (BAD, ONE, {}, dict(k=2 * MB + 8)), (BAD, ONE, {}, dict(k_stride=255)), (BAD, ONE, {}, dict(k_stride=260)), (BAD, ONE, {}, dict(v_stride=-256)),
    (BAD, ONE, {}, dict(v_stride=1 << 60)), (BAD, ONE, {}, dict(rows=-1)), (BAD, ONE, {}, dict(rows=1 << 60)), (BAD, ONE, {}, dict(k=16 * MB + 512)),
])
def test_refusals_of_rows(shim, write, want, seqs, pool, kw):
    assert rows_call(shim, seqs, pages(**pool), write, **kw) == want


def test_refusals_that_differ_between_writing_and_reading(shim):
    shared = [dict(n_q=3, n_kv=40), dict(q_row=2, n_q=2, n_kv=40)]
    assert rows_call(shim, shared, pages(), True) == OK and rows_call(shim, shared, pages(), False) == BAD
    table_in_rows = dict(table=2 * MB + 512)
    assert rows_call(shim, ONE, pages(), True, **table_in_rows) == OK and rows_call(shim, ONE, pages(), False, **table_in_rows) == BAD
    table_in_pool = dict(table=16 * MB + 512)
    assert rows_call(shim, ONE, pages(), True, **table_in_pool) == BAD and rows_call(shim, ONE, pages(), False, **table_in_pool) == OK
    same = dict(k=2 * MB, v=2 * MB)
    assert rows_call(shim, ONE, pages(), True, **same) == OK and rows_call(shim, ONE, pages(), False, **same) == BAD
    crossed = dict(k=2 * MB, v=2 * MB + 256, k_stride=512, v_stride=512)
    assert rows_call(shim, ONE, pages(), False, **crossed) == BAD
    unlike = dict(k=2 * MB, v=2 * MB + 512, k_stride=512, v_stride=1024)
    assert rows_call(shim, ONE, pages(), False, **unlike) == BAD


def attention_call(shim, seqs, pool, dtype=BF16, heads=(8, 4, 64), **kw):
    a = dict(pages=pool, table=1 * MB, table_stride=8, q=2 * MB, q_rows=100, window=mvla.WINDOW_ALL, n_sink=0, scale=0.0, out=3 * MB, workspace=64 * MB,
             workspace_bytes=1 << 40)
    a.update(kw)
    n = C.c_int64(-1)
    return shim.attention(dtype, *heads, len(seqs), mvla.c_seqs([mvla.Seq(**s) for s in seqs]), C.byref(mvla.CPagedAttention(**a)), C.byref(n)), n.value


@pytest.mark.parametrize("want,seqs,pool,kw", [
    (OK, ONE, {}, {}), (OK, ONE, KINDS["e4m3"], {}), (OK, ONE, KINDS["e2m1"], dict(lse=4 * MB)), (OK, MANY, KINDS["e4m3"], dict(q_rows=400, out=5 * MB)), (OK, [dict(n_q=0, n_kv=40)], {}, dict(q=None, out=None, table=None)),
    (OK, [dict(n_q=2, n_kv=0)], {}, dict(table=None)), (OK, [dict(n_q=1, n_kv=40), dict(q_row=1, n_q=1, n_kv=40)], {}, {}),
    (CAP, ONE * 5, {}, {}), (BAD, [], {}, {}), (BAD, [dict(n_q=-1, n_kv=40)], {}, {}), (BAD, [dict(q_row=98, n_q=3, n_kv=4)], {}, {}), (BAD, [dict(n_q=1, n_kv=513)], {}, {}),
    (BAD, [dict(n_q=2, n_kv=4), dict(q_row=1, n_q=2, n_kv=4)], {}, {}), (BAD, ONE, {}, dict(window=0)), (BAD, ONE, {}, dict(n_sink=-1)),
    (BAD, ONE, {}, dict(scale=-1.0)), (BAD, ONE, {}, dict(scale=float("inf"))), (BAD, ONE, {}, dict(scale=float("nan"))), (BAD, ONE, {}, dict(scale=1e-40)),
    (BAD, ONE, {}, dict(q=None)), (BAD, ONE, {}, dict(out=None)), (BAD, ONE, {}, dict(table=None)), (BAD, ONE, {}, dict(q=2 * MB + 8)), (BAD, ONE, {}, dict(out=2 * MB)),
    (BAD, ONE, {}, dict(out=16 * MB)), (BAD, ONE, KINDS["e4m3"], dict(out=48 * MB)), (BAD, ONE, {}, dict(out=1 * MB)), (BAD, ONE, {}, dict(lse=3 * MB)),
    (BAD, ONE, {}, dict(lse=4 * MB + 2)), (BAD, ONE, {}, dict(kv_len=4 * MB, lse=4 * MB)), (BAD, ONE, {}, dict(q_rows=-1)), (BAD, ONE, {}, dict(q_rows=1 << 60)),
    (BAD, ONE, dict(k=None), {}), (UNSUP, ONE, dict(page_rows=20), {}),
    (BAD, MANY, KINDS["e4m3"], dict(workspace=None, q_rows=400, out=5 * MB)), (BAD, MANY, KINDS["e4m3"], dict(workspace_bytes=100, q_rows=400, out=5 * MB)),
    (BAD, MANY, KINDS["e4m3"], dict(workspace=64 * MB + 16, q_rows=400, out=5 * MB)), (BAD, MANY, KINDS["e4m3"], dict(workspace=16 * MB, q_rows=400, out=5 * MB)),
])
def test_refusals_of_attention(shim, want, seqs, pool, kw):
    assert attention_call(shim, seqs, pages(**pool), **kw)[0] == want


@pytest.mark.parametrize("kind", [P.E4M3, P.E2M1])
def test_the_reference_rounds_to_the_nearest(kind):
    """Every value of the reference is the nearest one that its scale offers, by search over all of them."""
    g = torch.Generator().manual_seed(1)
    x = torch.randn(40, 64, generator=g) * torch.exp2(torch.randint(-40, 40, (40, 1), generator=g).float())
    x[3] = 0
    value, codes, byte = P.quantise(x, kind)
    if kind == P.E4M3:
        steps = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
        steps = steps[torch.isfinite(steps)]
    else:
        steps = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], dtype=torch.float64)
    scale = torch.exp2(byte.double() - 127)
    scale = scale.repeat_interleave(64 if kind == P.E4M3 else 32, -1).view(40, 64) if kind == P.E2M1 else scale[:, None].expand(40, 64)
    every = steps[None, None, :] * scale[..., None]
    best = (every - x.double()[..., None]).abs().amin(-1)
    assert torch.equal((value - x.double()).abs(), best)
    assert torch.equal(P.values(codes, byte, kind), value)
    big = x.double().unflatten(-1, (-1, 64 if kind == P.E4M3 else 32)).abs().amax(-1)
    top = P.FORMAT[kind][0]
    s = torch.exp2(byte.double() - 127).view(big.shape)
    assert (big <= top * s).all() and ((big > top * s / 2) | (big == 0)).all()
