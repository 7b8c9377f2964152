"""A cache in pages at the ends of what it accepts: heads that leave threads over, scales and queries of all sizes, values whose weight is next to nothing."""
import pytest
import torch

import page_util as P
from page_util import E2M1, E4M3, ROWS
from paper_2604_09244_b200 import mvla
from test_gpu_page import BF16, FP32, context, generator, same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", [ROWS, E4M3, E2M1])
@pytest.mark.parametrize("dtype,G,d,page_rows", [(BF16, 20, 128, 16), (BF16, 3, 128, 256), (FP32, 33, 64, 32), (BF16, 11, 256, 16)])
def test_heads_that_leave_threads_over(kind, dtype, G, d, page_rows):
    """The last page of the pool is read, each tensor alone and both."""
    gen = generator(G + d)
    ctx = context(dtype, G, G, d)
    pool = P.make_pool(gen, 3, G, page_rows, d, kind, dtype)
    n = 2 * page_rows
    table = torch.tensor([[0, 2]], dtype=torch.int32, device="cuda")
    seqs = [mvla.Seq(q_row=0, n_q=n, n_kv=n)]
    want = P.rows_of(pool, kind, table, 0, n, page_rows)
    out = lambda: torch.full((n, G, d), 9.0, dtype=dtype, device="cuda")
    for k, v in ((out(), out()), (out(), None), (None, out())):
        ctx.page_read(pool, seqs, table, k_out=k, v_out=v)
        torch.cuda.synchronize()
        for got, exact in zip((k, v), want):
            assert got is None or same(got.double(), exact)


def test_clusters_of_two_shapes_on_two_streams():
    """Calls whose CTAs together ask for more tensor memory than there is, side by side: each as if it ran alone."""
    gen = generator(9)
    calls = []
    for kind, H, G, d, sizes in ((E2M1, 32, 32, 64, ((130, 2900), (62, 3000))), (E4M3, 32, 32, 64, ((20, 600),) * 4), (ROWS, 24, 24, 64, ((20, 600),) * 4)):
        ctx = context(BF16, H, G, d)
        lengths = [n for _, n in sizes]
        table, n_pages = P.make_table(gen, lengths, 64)
        pool = P.make_pool(gen, n_pages, G, 64, d, kind, BF16)
        seqs, at = [], 0
        for n_q, n in sizes:
            seqs.append(mvla.Seq(q_row=at, n_q=n_q, n_kv=n))
            at += n_q
        q = torch.randn(at, H, d, generator=gen, device="cuda").to(BF16)
        calls.append((ctx, pool, seqs, table, q, ctx.page_attention(pool, seqs, table, q), torch.cuda.Stream()))
    torch.cuda.synchronize()
    outs = [[] for _ in calls]
    for _ in range(40):
        for (ctx, pool, seqs, table, q, _, stream), out in zip(calls, outs):
            with torch.cuda.stream(stream):
                out.append(ctx.page_attention(pool, seqs, table, q))
    torch.cuda.synchronize()
    for call, out in zip(calls, outs):
        assert all(torch.equal(x, call[5]) for x in out)
