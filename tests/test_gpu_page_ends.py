"""A cache in pages at the ends of what it accepts: heads that leave threads over, scales and queries of all sizes, values whose weight is next to nothing."""
import pytest
import torch

import page_util as P
from page_util import E2M1, E4M3, ROWS
from page_strict import check
from paper_2604_09244_b200 import mvla
from test_page_plan_cpu import PAGE_TILE, TOKEN, plan, shim  # noqa: F401
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


# (heads, key heads, elements, queries, rows) of calls over quantised pages, and the form that they take: tokens; tiles unpacked on the way, for one and two blocks of
# query rows; unpacked first
CALLS = [(8, 4, 64, 1, 300), (8, 2, 96, 4, 700), (8, 4, 64, 37, 300), (8, 4, 128, 60, 900), (4, 2, 256, 20, 500), (32, 8, 128, 50, 9000), (8, 4, 64, 200, 500)]


def form_of(shim, kind, H, G, d, n_q, n, **kw):
    """Whether weights meet the values in fp16, and the form."""
    p, _ = plan(shim, [(n_q, n)], kind=kind, heads=(H, G, d), **kw)
    return p["form"] == TOKEN or p["unpack"] > 0, (p["form"], p["unpack"])


def test_calls_take_every_form(shim):
    assert {form_of(shim, E4M3, *c)[1] for c in CALLS} == {(TOKEN, 0), (PAGE_TILE, 1), (PAGE_TILE, 2), (PAGE_TILE, 0)}


@pytest.mark.parametrize("kind", [ROWS, E4M3, E2M1])
@pytest.mark.parametrize("call", CALLS)
def test_scales_of_all_sizes(shim, call, kind):
    """Scores that are as good as zero, or whose queries or keys are far from one: rows that a mask hides stay hidden."""
    H, G, d, n_q, n = call
    gen = generator(n_q + d)
    ctx = context(BF16, H, G, d)
    table, n_pages = P.make_table(gen, [n], 32)
    pool = P.make_pool(gen, n_pages, G, 32, d, kind, BF16)
    seqs = [mvla.Seq(q_row=0, n_q=n_q, n_kv=n)]
    window = 150 if n < 1000 else 8400
    fp16, _ = form_of(shim, kind, *call, window=window)
    x = torch.randn(n_q, H, d, generator=gen, device="cuda")
    for size, scale in ((1.0, 1e-30), (1.0, 1e-36), (1.0, 1e-37), (1.0, 9e-39), (2.0 ** -112, 0.0), (2.0 ** -125, 0.0), (2.0 ** -60, 2.0 ** -70)):
        check(ctx, pool, kind, seqs, table, (x * size).to(BF16), 32, fp16, window=window, scale=scale)


@pytest.mark.parametrize("kind", [E4M3, E2M1])
@pytest.mark.parametrize("call", CALLS)
def test_tiles_of_nothing(shim, call, kind):
    """Whole tiles on pages outside the pool, or of rows of zeros as they are written, under the diagonal and at a window's edge, with queries of small elements."""
    H, G, d, n_q, n = call
    gen = generator(n_q + 2 * d)
    ctx = context(BF16, H, G, d)
    table, n_pages = P.make_table(gen, [n], 64)
    pool = P.make_pool(gen, n_pages, G, 64, d, kind, BF16)
    seqs = [mvla.Seq(q_row=0, n_q=n_q, n_kv=n)]
    last = (n - 1) // 64
    window = n % 64 + n_q + 80 if n < 1000 else n - 70
    edge = max(0, n - window) // 64
    pages = table[0, [last, edge]].long()
    zero = P.quantise(torch.zeros(1, d, device="cuda", dtype=BF16), kind)
    fp16, _ = form_of(shim, kind, *call, window=window)
    x = torch.randn(n_q, H, d, generator=gen, device="cuda")
    for outside in (True, False):
        if outside:
            table[0, [last, edge]] = -1
        else:
            table[0, [last, edge]] = pages.to(torch.int32)
            for codes, scale in ((pool.k, pool.k_scale), (pool.v, pool.v_scale)):
                P.bits(codes)[pages] = P.bits(zero[1])[0]
                scale[pages] = zero[2][0]
        for size in (2.0 ** -4, 2.0 ** -12, 2.0 ** -40):
            check(ctx, pool, kind, seqs, table, (x * size).to(BF16), 64, fp16, window=window)


def sized_pool(gen, kind, G, d, n, page_rows, k=None, v=None, wide=BF16):
    """(pool, table) of one sequence whose rows of keys and values [n, G, d] are random, times k and v."""
    table, n_pages = P.make_table(gen, [n], page_rows, spare=0)
    j = torch.arange(n, device="cuda")
    out = []
    for size in (k, v):
        x = torch.randn(n, G, d, generator=gen, device="cuda")
        rows = torch.zeros(n_pages, page_rows, G, d, device="cuda")
        rows[table[0].long()[j // page_rows], j % page_rows] = x if size is None else size(x, j[:, None, None])
        out.append(P.quantise(rows.transpose(1, 2).contiguous().to(wide), kind))
    return mvla.PagePool(out[0][1].contiguous(), out[1][1].contiguous(), out[0][2], out[1][2]), table


@pytest.mark.parametrize("kind", [ROWS, E4M3, E2M1])
@pytest.mark.parametrize("call", CALLS)
def test_large_values_of_little_weight(shim, call, kind):
    """The first rows, or one in 40, have values 2^24 to 2^110 larger than the others and scores far below them, to nearly nothing or to nothing at all."""
    H, G, d, n_q, n = call
    gen = generator(n_q + 3 * d)
    ctx = context(BF16, H, G, d)
    seqs = [mvla.Seq(q_row=0, n_q=n_q, n_kv=n)]
    fp16, _ = form_of(shim, kind, *call)
    q = torch.randn(n_q, H, d, generator=gen, device="cuda")
    q[..., 0] = 8
    for faint in (lambda j: j < 64, lambda j: j % 40 == 7, lambda j: (j >= 64) & (j < 100)):
        for size, low in ((2.0 ** 24, -64.0), (2.0 ** 30, -2000.0), (2.0 ** 110, -2000.0), (2.0 ** 24, 0.0)):
            keys = lambda x, j: torch.where(faint(j) & (torch.arange(d, device="cuda") == 0), low, x)  # noqa: B023, E731
            pool, table = sized_pool(gen, kind, G, d, n, 32, keys, lambda x, j: torch.where(faint(j), x * size, x))  # noqa: B023
            check(ctx, pool, kind, seqs, table, q.to(BF16), 32, fp16)


@pytest.mark.parametrize("kind", [ROWS, E4M3, E2M1])
@pytest.mark.parametrize("call", CALLS)
def test_values_of_all_sizes(shim, call, kind):
    """Values that grow and shrink from row to row, over the whole range of the scales, those of rows that are not seen yet among them; values near its lower end."""
    H, G, d, n_q, n = call
    gen = generator(n_q + 5 * d)
    ctx = context(BF16, H, G, d)
    seqs = [mvla.Seq(q_row=0, n_q=n_q, n_kv=n)]
    fp16, _ = form_of(shim, kind, *call)
    q = torch.randn(n_q, H, d, generator=gen, device="cuda").to(BF16)
    new = n - n_q                                              # the first query's row
    for e in (lambda j: (j - new).clamp(min=0) * (200.0 / max(n_q, 8)) - 100, lambda j: (j - new).clamp(min=0) * 1.5 - 20, lambda j: (n - j) * (200.0 / n) - 110,
              lambda j: j * (200.0 / n) - 110, lambda j: j * 0.0 - 108, lambda j: j % 2 * 180.0 - 100, lambda j: j % 3 * 13.0 - 20):
        pool, table = sized_pool(gen, kind, G, d, n, 64, None, lambda x, j: x * torch.exp2(e(j.float()).clamp(-110, 110)))  # noqa: B023
        check(ctx, pool, kind, seqs, table, q, 64, fp16)


@pytest.mark.parametrize("kind", [ROWS, E4M3, E2M1])
@pytest.mark.parametrize("call", CALLS)
def test_large_scores(shim, call, kind):
    """Scores from 2^10 to 2^120: where one row's decides, its values come out as they are; nothing leaves the numbers."""
    H, G, d, n_q, n = call
    gen = generator(n_q + 11 * d)
    ctx = context(BF16, H, G, d)
    seqs = [mvla.Seq(q_row=0, n_q=n_q, n_kv=n)]
    fp16, _ = form_of(shim, kind, *call)
    q = torch.randn(n_q, H, d, generator=gen, device="cuda")
    q[..., 0] = 8
    for at in (5, 10, 17, 24, 30, 60, 110):
        pool, table = sized_pool(gen, kind, G, d, n, 64, None, lambda x, j: x * torch.exp2(j % 3 * 20.0 - 40))
        check(ctx, pool, kind, seqs, table, q.to(BF16), 64, fp16, scale=2.0 ** at)
    # the scores of one row in 30 far above the others'
    for at in (10, 17, 24, 60):
        pool, table = sized_pool(gen, kind, G, d, n, 64, lambda x, j: torch.where((j % 30 == 11) & (torch.arange(d, device="cuda") == 0), 40.0 + j / 60, x), lambda x, j: x * torch.exp2(j % 5 * 2.0 - 4))
        check(ctx, pool, kind, seqs, table, q.to(BF16), 64, fp16, scale=2.0 ** at)


@pytest.mark.parametrize("kind", [ROWS, E4M3, E2M1])
@pytest.mark.parametrize("call", CALLS)
def test_keys_of_all_sizes(shim, call, kind):
    """Keys that grow from row to row, those of rows that are not seen yet among them, with queries and a scale that fit the first ones, the last ones or those between; one in 40 rows larger, orthogonal
    to the queries.  (No score leaves 32 bits.)"""
    H, G, d, n_q, n = call
    gen = generator(n_q + 7 * d)
    ctx = context(BF16, H, G, d)
    seqs = [mvla.Seq(q_row=0, n_q=n_q, n_kv=n)]
    fp16, _ = form_of(shim, kind, *call)
    q = torch.randn(n_q, H, d, generator=gen, device="cuda").to(BF16)
    q[..., 0] = 0
    new = n - n_q                                              # the first query's row
    for e, at in ((lambda j: (j - new).clamp(min=0) * (110.0 / max(n_q, 8)) - 100, 100.0), (lambda j: (j - new).clamp(min=0) * 1.5 - 20, 20.0), (lambda j: (n - j) * (200.0 / n) - 110, 0.0),
                  (lambda j: j * (110.0 / n) - 100, 100.0), (lambda j: j * 0.0 - 108, 108.0), (lambda j: j % 3 * 13.0 - 20, 20.0), (lambda j: j * 0.0 + 100, -100.0)):
        pool, table = sized_pool(gen, kind, G, d, n, 64, lambda x, j: x * torch.exp2(e(j.float()).clamp(-110, min(110, 105 - at))))  # noqa: B023
        check(ctx, pool, kind, seqs, table, q, 64, fp16, scale=0.3 * 2.0 ** at)
    for size in (2.0 ** 22, 2.0 ** 40, 2.0 ** 100):
        along = lambda x, j: torch.where(j % 40 == 7, (torch.arange(d, device="cuda") == 0) * size, x)  # noqa: B023, E731
        pool, table = sized_pool(gen, kind, G, d, n, 64, along)
        check(ctx, pool, kind, seqs, table, q, 64, fp16)


@pytest.mark.parametrize("kind", [ROWS, E4M3, E2M1])
@pytest.mark.parametrize("call", CALLS)
def test_queries_and_keys_of_unlike_sizes(shim, call, kind):
    """Scores of ordinary size whose factors are at the ends of their types: queries, keys, and the scale."""
    H, G, d, n_q, n = call
    gen = generator(n_q + 13 * d)
    ctx = context(BF16, H, G, d)
    seqs = [mvla.Seq(q_row=0, n_q=n_q, n_kv=n)]
    fp16, _ = form_of(shim, kind, *call)
    x = torch.randn(n_q, H, d, generator=gen, device="cuda")
    for query, key, scale in ((-118, 115, 0), (-110, 122, -12), (112, -110, 0), (120, -105, -15), (-100, -20, 120), (60, 60, -121), (-125, 122, 3), (122, -108, -14)):
        for spread in (0.0, 24.0):
            pool, table = sized_pool(gen, kind, G, d, n, 64, lambda x, j: x * torch.exp2(key + (j % 7 == 2) * -spread))  # noqa: B023
            check(ctx, pool, kind, seqs, table, (x * 2.0 ** query).to(BF16), 64, fp16, scale=0.3 * 2.0 ** scale)


@pytest.mark.parametrize("kind", [E4M3, E2M1])
@pytest.mark.parametrize("call", CALLS)
def test_the_least_scale_bytes(shim, call, kind):
    """Scales of 2^-127 to 2^-118, which rows are never given as they are written: what they stand for, in keys beside large queries, and in values."""
    H, G, d, n_q, n = call
    gen = generator(n_q + 17 * d)
    ctx = context(BF16, H, G, d)
    seqs = [mvla.Seq(q_row=0, n_q=n_q, n_kv=n)]
    fp16, _ = form_of(shim, kind, *call)
    x = (torch.randn(n_q, H, d, generator=gen, device="cuda") * 2.0 ** 114).to(BF16)
    for keys in (True, False):
        pool, table = sized_pool(gen, kind, G, d, n, 64)
        scale = pool.k_scale if keys else pool.v_scale
        scale.copy_(torch.randint(0, 10, scale.shape, generator=gen, device="cuda"))
        check(ctx, pool, kind, seqs, table, x if keys else x * 2.0 ** -114, 64, fp16)
    for large in (0.0, 2.0 ** 126):                            # queries that meet zeros alone, beside the largest keys
        pool, table = sized_pool(gen, kind, G, d, n, 64, lambda x, j: torch.where(torch.arange(d, device="cuda") < 32, x * 0, x * 2.0 ** 122))
        q = torch.zeros(n_q, H, d, device="cuda")
        q[..., 3] = large
        check(ctx, pool, kind, seqs, table, q.to(BF16), 64, fp16)


@pytest.mark.parametrize("kind", [ROWS, E4M3, E2M1])
@pytest.mark.parametrize("H,G,d,n_q,n", [(8, 4, 64, 1, 300), (4, 2, 128, 37, 300), (2, 2, 256, 90, 500)])
def test_ends_of_fp32_contexts(H, G, d, n_q, n, kind):
    """The same of fp32 rows, and of quantised ones beside fp32 queries: small and large scales, scores, keys and values; a tile on pages outside the pool."""
    gen = generator(n_q + 19 * d)
    ctx = context(FP32, H, G, d)
    seqs = [mvla.Seq(q_row=0, n_q=n_q, n_kv=n)]
    q = torch.randn(n_q, H, d, generator=gen, device="cuda")
    make = lambda k, v: sized_pool(gen, kind, G, d, n, 64, k, v, FP32)  # noqa: E731
    pool, table = make(None, None)
    for size, scale in ((1.0, 1e-36), (1.0, 9e-39), (2.0 ** -125, 0.0), (2.0 ** -60, 2.0 ** -70), (1.0, 2.0 ** 12), (1.0, 2.0 ** 24), (1.0, 2.0 ** 40), (1.0, 2.0 ** 100)):
        check(ctx, pool, kind, seqs, table, q * size, 64, False, scale=scale)
    table[0, n // 64] = -1
    check(ctx, pool, kind, seqs, table, q * 2.0 ** -40, 64, False)
    for v in (lambda x, j: torch.where(j < 64, x * 2.0 ** 60, x), lambda x, j: x * torch.exp2((j - (n - n_q)).clamp(min=0) * (160.0 / max(n_q, 8)) - 80), lambda x, j: x * 2.0 ** -108):
        pool, table = make(lambda x, j: torch.where((j < 64) & (torch.arange(d, device="cuda") == 0), -2000.0, x), v)
        q[..., 0] = 8
        check(ctx, pool, kind, seqs, table, q, 64, False)
    for query, key in ((-110, 110), (110, -110)):
        pool, table = make(lambda x, j: x * 2.0 ** key, None)  # noqa: B023
        check(ctx, pool, kind, seqs, table, q * 2.0 ** query, 64, False)


def test_idle_sequences_do_not_refuse_a_read():
    """Rows read without outputs: a sequence without rows of its own may stand anywhere behind the others'."""
    gen = generator(23)
    ctx = context()
    table, n_pages = P.make_table(gen, [40, 30], 16)
    pool = P.make_pool(gen, n_pages, 4, 16, 64, E4M3, BF16)
    k, v = ctx.page_read(pool, [mvla.Seq(q_row=0, n_q=40, n_kv=40), mvla.Seq(q_row=45, n_q=0, n_kv=30)], table)
    assert k.shape[0] == v.shape[0] == 45
    for got, want in zip((k, v), P.rows_of(pool, E4M3, table, 0, 40, 16)):
        assert same(got[:40].double(), want)


@pytest.mark.parametrize("kind,H,G,d,sizes", [(ROWS, 28, 4, 128, ((100, 66), (187, 365))), (E2M1, 24, 8, 192, ((4, 52), (168, 555), (183, 669), (78, 369))), (E4M3, 24, 8, 256, ((81, 651),)),
                                              (E4M3, 12, 4, 64, ((30, 3000), (9, 100)))])
def test_the_same_bits_every_time(kind, H, G, d, sizes):
    """Groups of heads that do not fill a tile of 128 rows: what lies in the rows that are left over, from whatever ran before, changes no bit."""
    gen = generator(29)
    ctx = context(BF16, H, G, d)
    table, n_pages = P.make_table(gen, [n for _, n in sizes], 64)
    pool = P.make_pool(gen, n_pages, G, 64, d, kind, BF16)
    seqs, at = [], 0
    for n_q, n in sizes:
        seqs.append(mvla.Seq(q_row=at, n_q=n_q, n_kv=n))
        at += n_q
    q = torch.randn(at, H, d, generator=gen, device="cuda").to(BF16)
    noise = (torch.randn(at, H, d, generator=gen, device="cuda") * 1e30).to(BF16)
    want = None
    for _ in range(30):
        lse = torch.empty(at, H, device="cuda")
        out = ctx.page_attention(pool, seqs, table, q, lse=lse, n_sink=1, scale=2.0)
        want = want or (out, lse)
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
        ctx.page_attention(pool, seqs, table, noise)


@pytest.mark.parametrize("kind", [E4M3, E2M1])
@pytest.mark.parametrize("call", CALLS[2:])
def test_scales_as_far_apart_as_a_tile_takes(shim, call, kind):
    """Rows behind the first query's own 2^4 to 2^24 larger, in keys and in values: what it sees keeps every bit, whichever way the tile is read."""
    H, G, d, n_q, n = call
    gen = generator(n_q + 31 * d)
    ctx = context(BF16, H, G, d)
    seqs = [mvla.Seq(q_row=0, n_q=n_q, n_kv=n)]
    fp16, _ = form_of(shim, kind, *call)
    q = torch.randn(n_q, H, d, generator=gen, device="cuda").to(BF16)
    for power in (4, 6, 7, 8, 9, 10, 12, 18, 20, 21, 22, 24):
        larger = lambda x, j: torch.where(j > n - n_q, x * 2.0 ** power, x)  # noqa: B023, E731
        for k, v in ((larger, None), (None, larger)):
            pool, table = sized_pool(gen, kind, G, d, n, 64, k, v)
            check(ctx, pool, kind, seqs, table, q, 64, fp16)
