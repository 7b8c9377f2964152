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
