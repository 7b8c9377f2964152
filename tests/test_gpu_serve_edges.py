"""The calls around the prune point where indexes, heads and positions are at their ends, and two at once."""
import pytest
import torch

import serve_util as R
from paper_2604_09244_b200 import mvla
from paper_2604_09244_b200.mvla import Seq
from test_gpu_serve import TYPES, attend_case, bits, check_attention, context, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32", "fp8"])
def test_rows_behind_the_first_four_gigabytes_of_a_cache(dtype):
    """Offsets of elements and bytes that pass 32 bits, in all three calls."""
    H = G = 32
    d, n = 256, 300
    rows = (1 << 32) // (G * d * TYPES[dtype].itemsize) + 2 * n
    base = rows - n - 8
    ctx = context(dtype, H, G, d, batch=2)
    gen = torch.Generator("cuda").manual_seed(1)
    wide = R.WIDE[TYPES[dtype]]
    k, v = (torch.empty(rows, G, d, dtype=TYPES[dtype], device="cuda") for _ in range(2))
    q0, k0, v0 = (randn(gen, n, h, d, dtype=wide) for h in (H, G, G))
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    freq = 10000.0 ** (-torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d)
    q, _, _ = ctx.qk_norm_rope(q0, k0, pos, freq, v=v0, k_out=k, v_out=v, out_rows=pos + base)
    z, size = R.rope(k0, pos, freq, None, True, 1e-6, False)
    assert bool(((k[base:base + n].double() - z).abs() <= R.rope_tolerance(z, size, TYPES[dtype], n)).all())
    assert torch.equal(bits(v[base:base + n]), bits(v0.to(TYPES[dtype])))
    for n_q in (1, 40):
        at = n - n_q
        mass = torch.zeros(rows, device="cuda")
        out = ctx.window_attention([Seq(q_row=at, n_q=n_q, kv_row=base, n_kv=n)], q, k, v, window=100, n_sink=2, mass=mass)
        r = R.attention([Seq(q_row=at, n_q=n_q, n_kv=n)], q, k[base:base + n], v[base:base + n], 100, 2)[0]
        assert bool(((out[at:].double() - r["out"]).abs() <= R.attention_tolerance(r, d, TYPES[dtype])).all())
        m = mass[base:base + n].double()
        assert bool(((m - r["mass"]).abs() <= R.mass_tolerance(r, d, n_q, H, m * 0)).all())
    kv_pos = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    kv_pos[base:base + n] = pos
    seqs = [Seq(kv_row=base, n_kv=n, budget=n // 2)]
    src = R.evict([Seq(n_kv=n, budget=n // 2)], pos.cpu(), mass[base:base + n].cpu(), 2, 10)[0]
    want = [bits(x)[base + torch.tensor(src, device="cuda")] for x in (k, v)]
    ctx.cache_evict(seqs, k, v, kv_pos, mass, n_sink=2, n_recent=10)
    for x, w in zip((k, v), want):
        assert torch.equal(bits(x)[base:base + n // 2], w)
    ctx.close()


@pytest.mark.parametrize("heads", [(16, 1, 64), (17, 1, 64), (34, 2, 64), (33, 1, 128), (40, 1, 96), (128, 1, 64)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32", "fp8"])
def test_attention_of_large_groups(dtype, heads):
    ctx = context(dtype, *heads)
    for i, (nq, nkv) in enumerate((([1, 1], [70, 300]), ([9], [130]), ([17], [17]), ([40, 3], [40, 65]))):
        args, mass, kept = attend_case(dtype, *heads, nq, nkv, 60, 2, "count", seed=i)
        check_attention(ctx, args, mass, kept)
    ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp32", "fp8"])
@pytest.mark.parametrize("n_q", [1, 50])
def test_attention_of_positions_at_the_end_of_their_type(dtype, n_q):
    top = 2 ** 31 - 1
    ctx = context(dtype, 4, 2, 64)
    for window, sinks in ((None, 0), (30, 2), (2 ** 31 - 2, 0), (1, top), (5, 0)):
        args, mass, kept = attend_case(dtype, 4, 2, 64, [n_q, n_q], [200, 70], window, sinks, "filled", seed=3)
        for s in args["seqs"]:
            q, c = args["q_pos"][s.q_row:s.q_row + s.n_q], args["kv_pos"][s.kv_row:s.kv_row + s.n_kv]
            far = top - 2 * s.n_kv - 4
            q += far
            q[0] = top
            c[c > 40] += far
        check_attention(ctx, args, mass, kept)
        # queries that see nothing, between others
        args["q_pos"][args["seqs"][0].q_row] = -(2 ** 31)
        check_attention(ctx, args, mass, kept)
    ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp32", "fp8"])
@pytest.mark.parametrize("n_q", [1, 60])
def test_attention_where_nobody_sees_anything(dtype, n_q):
    ctx = context(dtype, 4, 2, 64)
    args, mass, kept = attend_case(dtype, 4, 2, 64, [n_q, n_q], [200, 70], 10, 1, "filled", seed=3)
    args["kv_pos"].fill_(-1)
    args["k"].fill_(float("nan"))
    args["v"].fill_(float("nan"))
    check_attention(ctx, args, mass, kept)
    ctx.close()


@pytest.mark.parametrize("dtype,n_q", [("bf16", 1), ("bf16", 70), ("fp8", 1), ("fp8", 70), ("fp32", 70)])
def test_two_captured_calls_on_two_streams(dtype, n_q):
    """Each graph has its own workspace: replayed beside each other they give what they give alone."""
    ctx = context(dtype, 8, 2, 128)
    graphs, outs, wants = [], [], []
    for seed in (1, 2):
        args, mass, kept = attend_case(dtype, 8, 2, 128, [n_q] * 4, [3000, 70, 900, 2500], 2000, 4, "count", seed=seed)
        out, m = torch.zeros_like(args["q"], dtype=R.WIDE[kept]), mass.clone()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ctx.window_attention(**args, out=out, mass=m)
        g.replay()
        torch.cuda.synchronize()
        graphs.append((g, args))
        outs.append((out, m, mass))
        wants.append((out.clone(), m.clone()))
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(20):
        for out, m, mass in outs:
            out.zero_()
            m.copy_(mass)
        torch.cuda.synchronize()
        for s, (g, _) in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for (out, m, _), (o, w) in zip(outs, wants):
            assert torch.equal(out, o) and torch.equal(m, w)
    ctx.close()


def test_full_batches():
    """As many sequences as a context can have, some without queries, some without rows."""
    n = 64
    for dtype in ("bf16", "fp32", "fp8"):
        ctx = context(dtype, 4, 2, 64, batch=n)
        for q_of in (lambda b: b % 2, lambda b: 0 if b % 7 == 0 else 1 + b):
            nq, nkv = [q_of(b) for b in range(n)], [(b * 37) % 211 for b in range(n)]
            args, mass, kept = attend_case(dtype, 4, 2, 64, nq, nkv, 50, 2, "count", seed=8)
            check_attention(ctx, args, mass, kept)
        ctx.close()
    with pytest.raises(mvla.MvlaError):
        context("bf16", 4, 2, 64, batch=100000)


@pytest.mark.parametrize("pos", ["count", "kept", "filled"])
@pytest.mark.parametrize("n_q", [1, 3, 50, 300])
@pytest.mark.parametrize("dtype", ["bf16", "fp32", "fp8"])
def test_attention_beside_rows_that_no_query_sees(dtype, n_q, pos):
    """Cached rows outside every window, behind every query or between the windows of queries far apart may hold NaN and infinities."""
    ctx = context(dtype, 4, 2, 64)
    for window, sinks in ((20, 3), (100, 0), (1, 1)):
        args, mass, kept = attend_case(dtype, 4, 2, 64, [n_q, n_q], [n_q + 333, n_q + 70], window, sinks, pos, seed=n_q)
        if pos == "filled":                              # queries far apart, and rows behind all of them
            for s in args["seqs"]:
                args["q_pos"][s.q_row:s.q_row + s.n_q] = torch.linspace(0, 1.5 * s.n_kv, s.n_q, device="cuda").to(torch.int32)
        some = 0
        for b, s in enumerate(args["seqs"]):
            c = args["kv_pos"][s.kv_row:s.kv_row + s.n_kv] if args["kv_pos"] is not None else torch.arange(s.n_kv, device="cuda")
            p = args["q_pos"][s.q_row:s.q_row + s.n_q] if args["q_pos"] is not None else torch.arange(s.n_kv - s.n_q, s.n_kv, device="cuda")
            seen = (c[None] >= 0) & (c[None] <= p[:, None]) & ((p[:, None] - c[None] < window) | (c[None] < sinks))
            unseen = s.kv_row + torch.nonzero(~seen.any(0)).flatten()
            some += unseen.numel()
            for x in (args["k"], args["v"]):
                x[unseen] = float("nan")
                if dtype != "fp8":
                    x[unseen[::3]] = float("inf")
        assert some > 0
        check_attention(ctx, args, mass, kept)
    ctx.close()
