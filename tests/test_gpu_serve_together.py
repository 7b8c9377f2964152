"""Arguments of the calls around the prune point that are used together: lengths on the device and positions that are data, caches that grow between the
replays of a graph, cached rows that sequences share, caches without rows."""
import pytest
import torch

import serve_util as R
from paper_2604_09244_b200.mvla import Seq
from test_gpu_serve import attend_case, bits, check_attention, check_evict, context, evict_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pos", ["kept", "filled"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32", "fp8"])
def test_lengths_on_the_device_beside_positions(dtype, pos):
    for heads in ((8, 4, 128), (4, 2, 64)):
        ctx = context(dtype, *heads)
        for nq, nkv, lens in (([1, 1, 1, 1], [100, 100, 300, 20], [0, 57, 999, -3]), ([9, 40, 3], [64, 500, 40], [3, 129, 40]),
                              ([1, 1], [9000, 9000], [8191, 20])):
            for window, sinks in ((None, 0), (60, 2)):
                for m in (True, False):
                    args, mass, kept = attend_case(dtype, *heads, nq, nkv, window, sinks, pos, seed=9, lens=lens, mass=m)
                    check_attention(ctx, args, mass, kept)
        ctx.close()


@pytest.mark.parametrize("dtype,n_q", [("bf16", 1), ("bf16", 40), ("fp32", 1), ("fp8", 1), ("fp8", 40)])
def test_captured_steps_over_caches_that_grow(dtype, n_q):
    """A captured attention and eviction with positions and lengths on the device: the decode step that device lengths exist for."""
    H, G, d, room, budget = 8, 2, 128, 700, [300, 500]
    ctx = context(dtype, H, G, d)
    args, _, kept = attend_case(dtype, H, G, d, [n_q, n_q], [room, room], 200, 4, "filled", seed=1, mass=False)
    args["k"], args["v"] = (x.float().nan_to_num(0.5).to(kept) for x in (args["k"], args["v"]))
    start = [x.clone() for x in (args["k"], args["v"], args["kv_pos"])]
    seqs = args["seqs"]
    mass = torch.zeros(args["k"].shape[0], device="cuda")
    kv_len = torch.zeros(2, dtype=torch.int32, device="cuda")
    out = torch.zeros(args["q"].shape, dtype=R.WIDE[kept], device="cuda")
    new_len = torch.zeros(2, dtype=torch.int32, device="cuda")
    cut = [Seq(kv_row=s.kv_row, n_kv=s.n_kv, budget=b) for s, b in zip(seqs, budget)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.window_attention(**dict(args, kv_len=kv_len), out=out, mass=mass)
        ctx.cache_evict(cut, args["k"], args["v"], args["kv_pos"], mass, n_sink=4, n_recent=8, kv_len=kv_len, kv_len_out=new_len)
    for lens in ([300, 500], [301, 480], [700, 1], [699, 699], [0, 650]):
        for x, y in zip((args["k"], args["v"], args["kv_pos"]), start):
            bits(x).copy_(bits(y))
        mass.zero_()
        kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
        before = dict(args, **{n: args[n].clone() for n in ("k", "v", "kv_pos")}, kv_len=kv_len.clone())
        graph.replay()
        torch.cuda.synchronize()
        refs = R.attention(**before)
        grown = torch.zeros_like(mass)
        ctx.window_attention(**before, mass=grown)           # (the same numbers, bit for bit: what eviction went by)
        for s, r in zip(seqs, refs):
            o = out[s.q_row:s.q_row + s.n_q].double()
            assert bool(((o - r["out"]).abs() <= R.attention_tolerance(r, d, kept)).all())
            c = slice(s.kv_row, s.kv_row + r["n"])
            assert bool(((grown[c].double() - r["mass"]).abs() <= R.mass_tolerance(r, d, s.n_q, H, grown[c].double() * 0)).all())
        want = R.evict(cut, before["kv_pos"].cpu(), grown.cpu(), 4, 8, lens)
        assert new_len.tolist() == [len(w) for w in want]
        for s, src in zip(seqs, want):
            at, rows = s.kv_row + torch.tensor(src, dtype=torch.long, device="cuda"), slice(s.kv_row, s.kv_row + len(src))
            assert torch.equal(bits(args["k"])[rows], bits(before["k"])[at]) and torch.equal(bits(args["v"])[rows], bits(before["v"])[at])
            assert torch.equal(args["kv_pos"][rows], before["kv_pos"][at]) and torch.equal(mass[rows], grown[at])
    ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp32", "fp8"])
@pytest.mark.parametrize("n_q", [1, 5, 90])
def test_cached_rows_that_sequences_share(dtype, n_q):
    """A common prefix, read by three sequences of which one goes on behind it."""
    H, G, d = 4, 2, 128
    ctx = context(dtype, H, G, d)
    args, _, kept = attend_case(dtype, H, G, d, [n_q, n_q, n_q], [400, 1, 1], 150, 3, "count", seed=3, mass=False)
    a, b, c = args["seqs"]
    for s, n in ((b, 300), (c, 399)):
        s.kv_row, s.n_kv = a.kv_row, n
    b.kv_row, b.n_kv = a.kv_row + 7, 300                     # (begins inside the first one's rows)
    for window in (None, 150):
        check_attention(ctx, dict(args, window=window), None, kept)
    ctx.close()


def test_eviction_with_lengths_and_long_caches():
    """Lengths on the device that leave most of a long run unused, over the sizes at which a sequence gets more than one CTA."""
    ctx = context("bf16", 1, 1, 64)
    for n, lens, budget in ((9000, 100, 50), (40000, 4097, 4096), (40000, 39999, 1), (70000, 0, 5), (400000, 399999, 200000)):
        seqs, k, v, pos, mass = evict_case("bf16", 1, 64, [n, 33], [budget, 20], 3)
        kv_len = torch.tensor([lens, 33], dtype=torch.int32, device="cuda")
        check_evict(ctx, seqs, k, v, pos, mass, 0, 1, kv_len=kv_len, in_place=lens % 2 == 1)
    ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp32", "fp8"])
@pytest.mark.parametrize("n_q", [1, 40, 300])
def test_a_batch_without_cached_rows(dtype, n_q):
    """Queries before anything is cached: they see nothing, whether the cache has rows of nobody's or none at all."""
    ctx = context(dtype, 4, 2, 128)
    for mass in (True, False):
        args, weights, kept = attend_case(dtype, 4, 2, 128, [n_q, 1], [0, 0], None, 0, "count", seed=1, mass=mass)
        check_attention(ctx, args, weights, kept)
        none = dict(args, k=args["k"][:0], v=args["v"][:0], seqs=[Seq(q_row=s.q_row, n_q=s.n_q) for s in args["seqs"]])
        check_attention(ctx, none, None if weights is None else weights[:0], kept)
    ctx.close()
