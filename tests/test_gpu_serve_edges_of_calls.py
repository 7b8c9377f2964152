"""The calls around the prune point at the ends of what they accept, as a program makes them."""
import pytest
import torch

from test_gpu_serve import TYPES, attend_case, bits, check_attention, context, randn
import serve_util as R
from cuda.bindings import runtime as cudart
from paper_2604_09244_b200 import mvla
from paper_2604_09244_b200 import workloads as W
from paper_2604_09244_b200.mvla import Seq
from parity_util import device_tensors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32", "fp8"])
def test_rows_of_an_empty_batch_into_a_cache(dtype):
    """A batch without tokens goes the way of every other one: nothing is written."""
    H, G, d = 8, 2, 64
    ctx = context(dtype, H, G, d)
    gen = torch.Generator("cuda").manual_seed(1)
    wide = R.WIDE[TYPES[dtype]]
    qkv = randn(gen, 0, (H + 2 * G) * d, dtype=wide)
    q, k, v = (x.unflatten(1, (-1, d)) for x in qkv.split([H * d, G * d, G * d], 1))
    kc, vc = (randn(gen, 50, G, d, dtype=TYPES[dtype]) for _ in range(2))
    k0, v0 = kc.clone(), vc.clone()
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    freq = torch.ones(d // 2, dtype=torch.float64, device="cuda")
    q_out, ko, vo = ctx.qk_norm_rope(q, k, none, freq, v=v, k_out=kc, v_out=vc, out_rows=none)
    assert q_out.shape == (0, H, d) and ko is kc and vo is vc
    torch.cuda.synchronize()
    assert torch.equal(bits(kc), bits(k0)) and torch.equal(bits(vc), bits(v0))
    ctx.close()


@pytest.mark.parametrize("dtype,n_q", [("bf16", 1), ("bf16", 40), ("fp32", 1), ("fp32", 40), ("fp8", 1), ("fp8", 40)])
def test_attention_with_the_smallest_scale(dtype, n_q):
    """All logits are nothing: the mean of the visible values, and rows that are not seen stay out of it."""
    ctx = context(dtype, 4, 2, 128)
    for scale in (1e-38, 1e-30):
        args, mass, kept = attend_case(dtype, 4, 2, 128, [n_q, n_q], [n_q + 100, n_q], 60, 2, "filled", seed=1, scale=scale)
        check_attention(ctx, args, mass, kept)
    ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp32", "fp8"])
def test_eviction_from_a_cache_without_rows(dtype):
    """Nothing is cached yet: nothing moves, and no rows stay."""
    ctx = context(dtype, 2, 2, 64)
    k, v = (torch.zeros(0, 2, 64, device="cuda").to(TYPES[dtype]) for _ in range(2))
    pos, mass = torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(0, device="cuda")
    left = torch.full((2,), 7, dtype=torch.int32, device="cuda")
    for kv_len in (None, torch.tensor([3, -1], dtype=torch.int32, device="cuda")):
        ctx.cache_evict([Seq(budget=5), Seq(budget=9)], k, v, pos, mass, n_sink=1, n_recent=4, kv_len=kv_len, kv_len_out=left.fill_(7))
        assert left.tolist() == [0, 0]
    ctx.close()


def test_memory_that_runs_out_between_two_outputs():
    """The first output, and what the caller gave, are let go when there is no memory for the next one."""
    ctx = context("bf16", 32, 32, 128)
    rows = 16384                                             # 128 MB to an output
    q, k = (torch.zeros(rows, 32, 128, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    pos = torch.zeros(rows, dtype=torch.int32, device="cuda")
    freq = torch.ones(64, dtype=torch.float64, device="cuda")
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    total = torch.cuda.mem_get_info()[1]
    before = torch.cuda.memory_allocated()
    try:
        torch.cuda.set_per_process_memory_fraction((torch.cuda.memory_reserved() + (192 << 20)) / total)
        for _ in range(2):
            with pytest.raises(RuntimeError):
                ctx.qk_norm_rope(q, k, pos, freq)
            assert torch.cuda.memory_allocated() == before
        ctx.qk_norm_rope(q, None, pos, freq)                 # one output fits
    finally:
        torch.cuda.set_per_process_memory_fraction(1.0)
    assert torch.cuda.memory_allocated() == before
    ctx.qk_norm_rope(q, k, pos, freq)
    ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp32", "fp8"])
def test_norms_of_rows_of_zeros(dtype):
    """However small the constant is, a row of zeros stays one; the others are normed as if it were not there."""
    ctx = context(dtype, 4, 2, 64)
    gen = torch.Generator("cuda").manual_seed(2)
    wide = R.WIDE[TYPES[dtype]]
    q, k = randn(gen, 20, 4, 64, dtype=wide), randn(gen, 20, 2, 64, dtype=wide)
    q[3], k[7], q[5, 1] = 0, 0, 0
    pos = torch.arange(20, dtype=torch.int32, device="cuda")
    freq = 10000.0 ** (-torch.arange(0, 64, 2, device="cuda", dtype=torch.float64) / 64)
    for eps in (1e-300, 1e-45, 1e-39, 1e-6, 1e30, 1e300):
        qo, ko, _ = ctx.qk_norm_rope(q, k, pos, freq, eps=eps)
        for x, got in ((q, qo), (k, ko)):
            z, size = R.rope(x, pos, freq, None, True, eps, False)
            assert bool(((got.double() - z).abs() <= R.rope_tolerance(z, size, TYPES[dtype], 20)).all()), eps
    ctx.close()


def test_calls_that_enqueue_nothing_leave_the_overlap_of_prune_steps():
    """Steps with the promise of stable inputs are ordered by events of their own; after other work of the context they wait for all of it once more.
    A call that is refused or has nothing to do is no such work: the captured steps depend on one another as if it had not been made."""
    wl = W.small_workload(7, batch=2, D=256, H=4, d=64, dtype="bf16", n_txt=(9, 17), n_2d=(90, 130), n_3d=(80, 60), cold_start=0)
    dev = device_tensors(wl)
    rows = dev["hidden"].shape[0]
    q, k, v = dev["q"], dev["k"], dev["v"]
    pos = torch.zeros(rows, dtype=torch.int32, device="cuda")
    freq = torch.ones(32, dtype=torch.float64, device="cuda")
    weights = torch.zeros(rows, device="cuda")

    def refused(ctx):
        with pytest.raises(mvla.MvlaError):
            ctx.window_attention([Seq(n_q=rows + 1, n_kv=rows)], q, k, v)
        with pytest.raises(mvla.MvlaError):
            ctx.qk_norm_rope(q, None, pos, freq[:5])
        with pytest.raises(mvla.MvlaError):
            ctx.cache_evict([Seq(n_kv=10, budget=5)], k, v, pos, weights, n_sink=4, n_recent=4)

    def empty(ctx):
        ctx.qk_norm_rope(q[:0], None, pos[:0], freq)
        ctx.window_attention([Seq(n_kv=rows)], q, k, v)

    def work(ctx):
        ctx.qk_norm_rope(q, None, pos, freq, q_out=torch.empty_like(q))

    def dependencies(between):
        ctx = mvla.context_for(wl)
        outs = [ctx.alloc_outputs(wl.samples, extras=True) for _ in range(11)]      # (a step in flight that writes the same buffers would be waited for)

        def step(i):
            ctx.prune_step(0, wl.samples, wl.mode, q, k, v, dev["hidden"], flags=mvla.FLAG_INPUTS_STABLE, out=outs[i])
        for i in range(8):
            step(i)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph(keep_graph=True)
        with torch.cuda.graph(graph):
            for i in range(8):
                step(i)
            between(ctx)
            for i in range(8, 11):
                step(i)
        raw = graph.raw_cuda_graph()
        rc, _, n = cudart.cudaGraphGetNodes(raw)
        rc, nodes, n = cudart.cudaGraphGetNodes(raw, n)
        place = {int(x): i for i, x in enumerate(nodes)}
        edges = cudart.cudaGraphGetEdges_v2(raw, cudart.cudaGraphGetEdges_v2(raw)[-1])
        ctx.close()
        return n, sorted((place[int(a)], place[int(b)]) for a, b in zip(edges[1], edges[2]))
    plain = dependencies(lambda ctx: None)
    assert plain[0] >= 22 and dependencies(refused) == plain and dependencies(empty) == plain
    assert dependencies(work) != plain
