"""Which form a call on a cache in pages takes, how it is cut, and that the tiles which kernels unpack lie inside the workspace: host arithmetic
(csrc/page_checks.h) against what the kernels compute of it, without a GPU."""
import ctypes as C
import os
import random
import subprocess

import pytest

import page_util
from paper_2604_09244_b200 import mvla

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SHIM = r"""
#include "page_checks.h"
using namespace mvla;
extern "C" void plan(int dtype, int H, int G, int d, int32_t n, const mvla_seq* s, const mvla_paged_attention* a, int64_t* out, int64_t* parts)
{
    const ServeShape v = {dtype, dtype == 1 ? 1 : 0, H, G, d, 64, 148, size_t(dtype == 1 ? 4 : 2), size_t(dtype == 1 ? 4 : 2)};
    const PageAttendPlan p = plan_page_attention(v, n, s, a);
    const AttendPlan& q = p.attend;
    const int64_t all[] = {q.form, p.unpack, q.cluster, q.part_keys, q.blocks, q.splits, q.rows, q.queries, q.part_o, q.part_ml, q.bytes, p.dense_tiles, p.dense_k, p.dense_v, p.bytes};
    for (int i = 0; i < 15; ++i) out[i] = all[i];
    for (int b = 0; b < n; ++b) {
        parts[2 * b] = parts_of(q, s[b], !a->kv_len, a->window, a->n_sink);
        parts[2 * b + 1] = seen_tiles(s[b], a->window, a->n_sink);
    }
}
"""
NAMES = ("form", "unpack", "cluster", "part_keys", "blocks", "splits", "rows", "queries", "part_o", "part_ml", "attend_bytes", "dense_tiles", "dense_k", "dense_v", "bytes")
FMA, TILE, TOKEN, PAGE_TILE = range(4)
ROWS, E4M3, E2M1 = mvla.PAGE_ROWS, mvla.PAGE_E4M3, mvla.PAGE_E2M1
BF16, FP32 = mvla.DTYPE_BF16, mvla.DTYPE_FP32


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    d = tmp_path_factory.mktemp("shim")
    src, lib = str(d / "shim.cpp"), str(d / "shim.so")
    open(src, "w").write(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_2604_09244_b200", "csrc"), src, "-o", lib], check=True)
    return C.CDLL(lib)


def plan(shim, seqs, kind=E4M3, dtype=BF16, heads=(32, 8, 128), window=mvla.WINDOW_ALL, n_sink=0, kv_len=None):
    a = mvla.CPagedAttention(pages=mvla.CPages(n_pages=10, page_rows=64, kind=kind), window=window, n_sink=n_sink, kv_len=kv_len)
    out, parts = (C.c_int64 * 15)(), (C.c_int64 * (2 * len(seqs)))()
    shim.plan(dtype, *heads, len(seqs), mvla.c_seqs([mvla.Seq(n_q=q, n_kv=n) for q, n in seqs]), C.byref(a), out, parts)
    return dict(zip(NAMES, out)), [tuple(parts[2 * i:2 * i + 2]) for i in range(len(seqs))]


@pytest.mark.parametrize("want,kw", [
    ((TOKEN, 0), dict(seqs=[(1, 4000)])), ((TOKEN, 0), dict(seqs=[(4, 60000)], kind=E2M1)), ((PAGE_TILE, 1), dict(seqs=[(5, 60000)])),
    ((PAGE_TILE, 2), dict(seqs=[(64, 9000), (1, 4000)])), ((PAGE_TILE, 1), dict(seqs=[(64, 20000)], heads=(16, 4, 256))), ((PAGE_TILE, 0), dict(seqs=[(64, 9000)] + [(1, 9)] * 9)),
    ((PAGE_TILE, 0), dict(seqs=[(64, 8000)])), ((PAGE_TILE, 0), dict(seqs=[(65, 4000)])), ((PAGE_TILE, 0), dict(seqs=[(65, 4000)], kind=ROWS)),
    ((TOKEN, 0), dict(seqs=[(1, 800)], kind=ROWS)), ((PAGE_TILE, 0), dict(seqs=[(1, 8000)], kind=ROWS)), ((TOKEN, 0), dict(seqs=[(4, 200)], kind=ROWS)),
    ((TOKEN, 0), dict(seqs=[(4, 1200)] * 4, kind=ROWS)), ((PAGE_TILE, 0), dict(seqs=[(4, 200)] * 40, kind=ROWS)), ((TOKEN, 0), dict(seqs=[(2, 200)] * 40, kind=ROWS)), ((TOKEN, 0), dict(seqs=[(4, 4000)], kind=ROWS, heads=(32, 8, 64))), ((PAGE_TILE, 0), dict(seqs=[(4, 5000)], kind=ROWS, heads=(32, 8, 64))),
    ((TOKEN, 0), dict(seqs=[(1, 60000)], kind=ROWS, heads=(32, 8, 64))), ((PAGE_TILE, 0), dict(seqs=[(5, 200)], kind=ROWS)), ((PAGE_TILE, 0), dict(seqs=[(4, 200)], kind=ROWS, heads=(32, 8, 256))),
    ((TOKEN, 0), dict(seqs=[(2, 60000)], kind=ROWS, heads=(32, 8, 96))), ((PAGE_TILE, 0), dict(seqs=[(3, 60000)], kind=ROWS, heads=(32, 8, 96))),
    ((PAGE_TILE, 0), dict(seqs=[(1, 8000)], kind=ROWS, heads=(16, 2, 256))), ((TOKEN, 0), dict(seqs=[(1, 300)] * 30 + [(0, 90000)], kind=ROWS, heads=(16, 16, 256))),
    ((PAGE_TILE, 2), dict(seqs=[(5, 80000)], heads=(64, 1, 64))), ((FMA, 0), dict(seqs=[(1, 800)], dtype=FP32)), ((FMA, 0), dict(seqs=[(300, 800)], dtype=FP32, kind=ROWS)),
])
def test_forms(shim, want, kw):
    p, _ = plan(shim, **kw)
    assert (p["form"], p["unpack"]) == want
    dense = p["form"] != TOKEN and not p["unpack"] and kw.get("kind", E4M3) != ROWS
    assert (p["dense_tiles"] > 0) == dense and (p["dense_k"] >= 0) == dense


def counted_tiles(n, lo, hi, window, n_sink):
    """(sinks, first, count) of tiles of 64 keys that queries at [lo, hi] see of n cached rows, as the kernels count them."""
    end = -(-(min(n - 1, max(hi, -1)) + 1) // 64)
    first = min((0 if window > lo else lo - window + 1) // 64, end)
    sinks = min(-(-n_sink // 64), first)
    return sinks, first, sinks + end - first


@pytest.mark.parametrize("seed", range(4))
def test_unpacked_tiles_lie_inside_the_workspace(shim, seed):
    rng = random.Random(seed)
    for _ in range(400):
        dtype = rng.choice([BF16, FP32])
        seqs = [(rng.choice([0, 1, rng.randint(1, 500)]), rng.randint(0, 3000)) for _ in range(rng.randint(1, 5))]
        window, n_sink = rng.choice([mvla.WINDOW_ALL, rng.randint(1, 2000), 1]), rng.choice([0, 1, rng.randint(0, 300)])
        p, per = plan(shim, seqs + [(300, 10)], dtype=dtype, heads=(8, 4, 64), window=window, n_sink=n_sink, kv_len=4096)
        assert p["dense_tiles"] == sum(t for _, t in per)
        assert p["dense_v"] >= p["dense_k"] + p["dense_tiles"] * 64 * 4 * 64 * (4 if dtype == FP32 else 2)
        kernel_sinks = 1 if window == mvla.WINDOW_ALL and n_sink == 0 else n_sink
        for (n_q, n_kv), (_, tiles) in zip(seqs, per):
            if n_q == 0:
                continue
            for n in {n_kv, rng.randint(0, n_kv), 0}:            # lengths on the device
                pos = lambda i: max(n - n_q + i, -1)  # noqa: E731
                sinks, first, count = counted_tiles(n, pos(0), pos(n_q - 1), window, kernel_sinks)
                assert count <= tiles
                for q0 in range(0, n_q, 64):                     # a block's tiles, where the sequence's lie
                    s, f, c = counted_tiles(n, pos(q0), pos(min(q0 + 64, n_q) - 1), window, kernel_sinks)
                    for t in range(c):
                        tile = t if t < s else f + t - s
                        place = tile if tile < sinks else tile - first + sinks
                        assert 0 <= place < count


@pytest.mark.parametrize("seed", range(4))
def test_parts_cover_and_fit(shim, seed):
    rng = random.Random(seed + 10)
    for _ in range(300):
        heads = rng.choice([(32, 8, 128), (8, 8, 64), (16, 16, 256), (28, 4, 128), (64, 1, 64)])
        kind = rng.choice([ROWS, E4M3, E2M1])
        most = rng.choice([1, 2, 100])
        seqs = [(rng.randint(0, most), rng.choice([0, 1, rng.randint(1, 1 << rng.randint(1, 20))])) for _ in range(rng.choice([1, 3, 64]))]
        p, per = plan(shim, seqs, kind=kind, heads=heads)
        assert p["cluster"] in (1, 2, 4, 8)
        if p["form"] == FMA or not any(q for q, _ in seqs):
            continue
        results = 0
        for (q, n), (parts, _) in zip(seqs, per):
            assert parts == (0 if q == 0 else max(1, -(-n // p["part_keys"]))) and parts <= 256
            results += q * parts
        assert p["splits"] == max(parts for parts, _ in per)
        if p["splits"] > 1:
            assert p["part_ml"] >= p["part_o"] + results * heads[0] * heads[2] * 4 and p["attend_bytes"] >= p["part_ml"] + results * heads[0] * 8


@pytest.mark.parametrize("seed", range(4))
def test_fp32_parts_fit(shim, seed):
    rng = random.Random(seed + 20)
    for _ in range(300):
        heads = rng.choice([(32, 8, 128), (8, 8, 64), (16, 16, 256), (28, 4, 96), (64, 1, 64)])
        seqs = [(rng.randint(0, rng.choice([1, 3, 400])), rng.choice([0, 1, rng.randint(1, 1 << rng.randint(1, 20))])) for _ in range(rng.choice([1, 3, 64]))]
        kind = rng.choice([ROWS, E4M3])
        p, per = plan(shim, seqs, kind=kind, dtype=FP32, heads=heads)
        assert p["form"] == FMA and 1 <= p["splits"] <= 64
        for (q, _), (parts, _) in zip(seqs, per):
            assert parts == (p["splits"] if q else 0)
        if p["splits"] > 1:
            results = p["splits"] * sum(q for q, _ in seqs)
            assert p["part_ml"] >= p["part_o"] + results * heads[0] * heads[2] * 4 and p["attend_bytes"] >= p["part_ml"] + results * heads[0] * 8
            assert kind == ROWS or p["dense_k"] < 0 or p["dense_k"] >= p["attend_bytes"]


@pytest.mark.parametrize("call", list(page_util.CLUSTERS))
def test_clusters(shim, call):
    kind, H, G, d, seqs = call
    p, _ = plan(shim, list(seqs), kind=kind, heads=(H, G, d))
    assert (p["form"], p["unpack"], p["cluster"], p["splits"] > 1) == (PAGE_TILE, *page_util.CLUSTERS[call])
