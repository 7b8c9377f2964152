"""A cache in pages where a kernel can go wrong: offsets past 32 bits, scales far apart, lengths on the device, captured calls, batches and pools
that are empty, many query rows to a key head, and what the binding refuses."""
import pytest
import torch

import page_util as P
import serve_util as U
from page_util import E2M1, E4M3, ROWS
from paper_2604_09244_b200 import mvla
from test_gpu_page import check_attention, context, generator, same

pytestmark = pytest.mark.gpu
BF16, FP32, FP8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
KINDS = [ROWS, E4M3, E2M1]


def some_pages(ctx, gen, kind, G, d, page_rows, lengths, wide=BF16):
    table, n_pages = P.make_table(gen, lengths, page_rows)
    return table, P.make_pool(gen, n_pages, G, page_rows, d, kind, wide)


@pytest.mark.parametrize("kind", KINDS)
def test_offsets_past_32_bits(kind):
    """Pools of more than 2^32 bytes a tensor, pages at their end."""
    gen = generator(1)
    G, d, page_rows, n = 8, 128, 256, 700
    ctx = context(BF16, 16, G, d)
    row = {ROWS: 2 * d, E4M3: d, E2M1: d // 2}[kind]
    n_pages = (2 ** 32 + 2 ** 28) // (G * page_rows * row)
    shape = (n_pages, G, page_rows)
    data = lambda: torch.empty(*shape, row, dtype=torch.uint8, device="cuda").view({ROWS: BF16, E4M3: FP8, E2M1: torch.uint8}[kind])  # noqa: E731
    scale = lambda: None if kind == ROWS else torch.empty(*shape, *([] if kind == E4M3 else [d // 32]), dtype=torch.uint8, device="cuda")  # noqa: E731
    pool = mvla.PagePool(data(), data(), scale(), scale())
    table = torch.tensor([[n_pages - 1, 3, n_pages - 2]], dtype=torch.int32, device="cuda")
    new = torch.randn(n, 2, G, d, generator=gen, device="cuda").to(BF16)
    seqs = [mvla.Seq(q_row=0, n_q=n, n_kv=n)]
    ctx.page_write(pool, seqs, table, new[:, 0], new[:, 1])
    k, v = ctx.page_read(pool, seqs, table)
    assert same(k.double(), P.quantise(new[:, 0], kind)[0]) and same(v.double(), P.quantise(new[:, 1], kind)[0])
    for n_q in (1, 6, 90):
        q = torch.randn(n_q, 16, d, generator=gen, device="cuda").to(BF16)
        check_attention(ctx, pool, kind, [mvla.Seq(q_row=0, n_q=n_q, n_kv=n)], table, q, page_rows)


@pytest.mark.parametrize("n_q", [1, 4, 6, 70, 300])
@pytest.mark.parametrize("kind", [E4M3, E2M1])
def test_scales_far_apart(kind, n_q):
    """Rows of keys and of values whose sizes differ by 2^18: nothing is lost of them but what their weights round to."""
    gen = generator(n_q)
    H, G, d, page_rows, n = 8, 4, 128, 32, 900
    ctx = context(BF16, H, G, d)
    table, n_pages = P.make_table(gen, [n], page_rows)
    out = []
    for _ in range(2):
        x = torch.randn(n_pages, G, page_rows, d, generator=gen, device="cuda") * torch.exp2(torch.randint(-9, 10, (n_pages, G, page_rows, 1), generator=gen, device="cuda").float())
        if kind == E2M1:
            x = x.unflatten(-1, (-1, 32)) * torch.exp2(torch.randint(-3, 1, (n_pages, G, page_rows, 4, 1), generator=gen, device="cuda").float())
            x = x.flatten(-2)
        out.append(P.quantise(x.to(BF16), kind)[1:])
    pool = mvla.PagePool(out[0][0].contiguous(), out[1][0].contiguous(), out[0][1].contiguous(), out[1][1].contiguous())
    q = (torch.randn(n_q, H, d, generator=gen, device="cuda") * 2.0 ** -7).to(BF16)
    check_attention(ctx, pool, kind, [mvla.Seq(q_row=0, n_q=n_q, n_kv=n)], table, q, page_rows)


@pytest.mark.parametrize("n_q", [1, 6, 70, 300])
@pytest.mark.parametrize("kind", [E4M3, E2M1])
def test_tiles_of_growing_values(kind, n_q):
    """Every 64 rows' values are 2^9 larger than the ones before, up to 2^100, and what a query sees last decides; then the other way round.  Rows of zeros between."""
    gen = generator(n_q + 50)
    H, G, d, page_rows, n = 4, 4, 64, 64, 64 * 12
    ctx = context(BF16, H, G, d)
    for down in (False, True):
        table, n_pages = P.make_table(gen, [n], page_rows, spare=0)
        size = torch.zeros(n_pages, device="cuda")
        order = torch.arange(12, device="cuda").float()
        size[table[0].long()] = (11 - order if down else order) * 9 - 4
        v = torch.randn(n_pages, G, page_rows, d, generator=gen, device="cuda") * torch.exp2(size)[:, None, None, None]
        v[:, :, 5] = 0
        k = torch.randn(n_pages, G, page_rows, d, generator=gen, device="cuda")
        k[:, :, 9] = 0
        kq, vq = P.quantise(k.to(BF16), kind), P.quantise(v.to(BF16), kind)
        pool = mvla.PagePool(kq[1].contiguous(), vq[1].contiguous(), kq[2].contiguous(), vq[2].contiguous())
        seqs = [mvla.Seq(q_row=0, n_q=n_q, n_kv=n)]
        q = torch.randn(n_q, H, d, generator=gen, device="cuda").to(BF16)
        # (summed by size: nothing of the faint values is left beside the largest, and nothing has to be)
        check_attention(ctx, pool, kind, seqs, table, q, page_rows)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n_q", [1, 7, 80])
def test_queries_of_all_sizes(kind, n_q):
    """Rows of queries from 2^-100 to 2^100 with keys and a scale that fit them; rows of zeros."""
    gen = generator(7)
    H, G, d, page_rows, n = 8, 4, 96, 16, 400
    ctx = context(BF16, H, G, d)
    table, pool = some_pages(ctx, gen, kind, G, d, page_rows, [n])
    q = torch.randn(n_q, H, d, generator=gen, device="cuda")
    for factor in (2.0 ** -100, 2.0 ** 100, 2.0 ** -30):
        x = (q * factor).to(BF16)
        x[0, 1] = 0
        check_attention(ctx, pool, kind, [mvla.Seq(q_row=0, n_q=n_q, n_kv=n)], table, x, page_rows, scale=0.1 / factor)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_lengths_on_the_device(kind, dtype):
    gen = generator(8)
    H, G, d, page_rows = 8, 4, 64, 32
    ctx = context(dtype, H, G, d)
    most = 700
    table, pool = some_pages(ctx, gen, kind, G, d, page_rows, [most] * 6, wide=dtype)
    for n_q in (1, 5, 70):
        seqs = [mvla.Seq(q_row=80 * b, n_q=n_q, n_kv=most) for b in range(6)]
        kv_len = torch.tensor([700, 0, 1, 33, 5000, -7], dtype=torch.int32, device="cuda")      # (taken into [0, 700])
        q = torch.randn(480, H, d, generator=gen, device="cuda").to(dtype)
        check_attention(ctx, pool, kind, seqs, table, q, page_rows, kv_len=kv_len)
        check_attention(ctx, pool, kind, seqs, table, q, page_rows, kv_len=kv_len, window=20, n_sink=3)


@pytest.mark.parametrize("kind", KINDS)
def test_many_rows_to_a_key_head(kind):
    """64 and 40 query heads to one key head: a single token is a block of rows."""
    gen = generator(9)
    for H, G, d in ((64, 1, 64), (40, 1, 128), (34, 2, 64)):
        ctx = context(BF16, H, G, d)
        lengths = [1, 130, 2000]
        table, pool = some_pages(ctx, gen, kind, G, d, 64, lengths)
        for n_q in (1, 9):
            seqs = [mvla.Seq(q_row=9 * i, n_q=n_q, n_kv=n) for i, n in enumerate(lengths)]
            q = torch.randn(27, H, d, generator=gen, device="cuda").to(BF16)
            check_attention(ctx, pool, kind, seqs, table, q, 64)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n_q,n,window", [(5, 9000, None), (33, 5000, None), (64, 20000, 3000), (2, 40000, None), (1, 70000, 50000), (300, 4000, None)])
def test_parts_of_long_sequences(kind, n_q, n, window):
    gen = generator(n_q)
    H, G, d, page_rows = 8, 2, 128, 64
    ctx = context(BF16, H, G, d)
    lengths = [n, 100, n // 3]
    table, pool = some_pages(ctx, gen, kind, G, d, page_rows, lengths)
    seqs = [mvla.Seq(q_row=0, n_q=n_q, n_kv=n), mvla.Seq(q_row=n_q, n_q=min(n_q, 7), n_kv=100), mvla.Seq(q_row=2 * n_q, n_q=n_q, n_kv=n // 3)]
    q = torch.randn(3 * n_q, H, d, generator=gen, device="cuda").to(BF16)
    a = check_attention(ctx, pool, kind, seqs, table, q, page_rows, window=window, n_sink=70)
    b = check_attention(ctx, pool, kind, seqs, table, q, page_rows, window=window, n_sink=70)
    assert torch.equal(a, b)                                   # no order that changes from run to run


@pytest.mark.parametrize("kind", KINDS)
def test_full_batch_of_unlike_sequences(kind):
    gen = generator(11)
    H, G, d, page_rows = 4, 2, 64, 16
    ctx = context(BF16, H, G, d, batch=64)
    lengths = [(i * 37) % 211 for i in range(64)]
    table, pool = some_pages(ctx, gen, kind, G, d, page_rows, lengths)
    for shape in (lambda i: 1 if i % 5 else 0, lambda i: (i * 7) % 40):
        row, seqs = 0, []
        for i, n in enumerate(lengths):
            seqs.append(mvla.Seq(q_row=row, n_q=shape(i), n_kv=n))
            row += shape(i)
        q = torch.randn(row, H, d, generator=gen, device="cuda").to(BF16)
        check_attention(ctx, pool, kind, seqs, table, q, page_rows, window=50, n_sink=1)


def test_a_token_beside_a_chunk_keeps_its_bits():
    """Unquantised pages: single tokens' weights keep 16 bits whatever else is in the batch."""
    gen = generator(12)
    H, G, d, page_rows = 8, 4, 128, 32
    ctx = context(BF16, H, G, d)
    lengths = [3000, 500]
    table, pool = some_pages(ctx, gen, ROWS, G, d, page_rows, lengths)
    seqs = [mvla.Seq(q_row=0, n_q=1, n_kv=3000), mvla.Seq(q_row=1, n_q=100, n_kv=500)]
    q = torch.randn(101, H, d, generator=gen, device="cuda").to(BF16)
    out = check_attention(ctx, pool, ROWS, seqs, table, q, page_rows)
    r = P.attention(pool, ROWS, seqs[:1], table, q, page_rows)[0]
    own = (2 * U.logit_error(r["reach"], d) + 2.0 ** -20 + 2 * r["keys"] * 2.0 ** -24 + 2.0 ** -16)[..., None] * r["weight"]
    assert ((out[:1].double() - r["out"]).abs() <= own + U.HALF[BF16] * (r["out"].abs() + own)).all()


@pytest.mark.parametrize("kind", KINDS)
def test_nothing_to_see_and_nothing_to_do(kind):
    gen = generator(13)
    H, G, d = 8, 4, 64
    for dtype in (BF16, FP32):
        ctx = context(dtype, H, G, d)
        empty = ctx.alloc_pages(0, page_rows=16, kind=kind)
        for n_q in (1, 50):
            q = torch.randn(n_q, H, d, generator=gen, device="cuda").to(dtype)
            lse = torch.zeros(n_q, H, device="cuda")
            # no cached rows; a pool without pages (zeros)
            out = ctx.page_attention(empty, [mvla.Seq(n_q=n_q, n_kv=0)], torch.empty(1, 0, dtype=torch.int32, device="cuda"), q, lse=lse)
            assert (out == 0).all() and (lse == float("-inf")).all()
            table = torch.zeros(1, 9, dtype=torch.int32, device="cuda")
            out = ctx.page_attention(empty, [mvla.Seq(n_q=n_q, n_kv=130)], table, q, lse=lse)
            seen = (130 - n_q + 1 + torch.arange(n_q, device="cuda")).float().log()
            assert (out == 0).all() and ((lse - seen[:, None]).abs() <= 2.0 ** -18).all()
        k, v = ctx.page_read(empty, [mvla.Seq(n_q=20, n_kv=20)], torch.zeros(1, 2, dtype=torch.int32, device="cuda"))
        assert (k == 0).all() and (v == 0).all()
        ctx.page_write(empty, [mvla.Seq(n_q=20, n_kv=20)], torch.zeros(1, 2, dtype=torch.int32, device="cuda"), k, v)
        pool = ctx.alloc_pages(2, page_rows=16, kind=kind)
        none = torch.empty(0, G, d, dtype=ctx.hidden_dtype, device="cuda")
        table = torch.zeros(1, 2, dtype=torch.int32, device="cuda")
        ctx.page_write(pool, [mvla.Seq(n_q=0, n_kv=20)], table, none, none)
        k, v = ctx.page_read(pool, [mvla.Seq(n_q=0, n_kv=20)], table)
        assert k.shape == (0, G, d)
        out = ctx.page_attention(pool, [mvla.Seq(n_q=0, n_kv=20)], table, torch.empty(0, H, d, dtype=ctx.hidden_dtype, device="cuda"))
        assert out.shape == (0, H, d)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype,n_q", [(BF16, 1), (BF16, 40), (FP32, 3)])
def test_captured_and_growing(kind, dtype, n_q):
    """A step's write and attention in a graph, replayed as the caches grow; a second graph of the same calls runs beside it on a stream of its own."""
    gen = generator(14)
    H, G, d, page_rows, most, steps = 8, 4, 64, 16, 400, 4
    ctx = context(dtype, H, G, d)
    runs = []
    for b in range(2):
        table, n_pages = P.make_table(gen, [most, most], page_rows)
        r = {"pool": P.make_pool(gen, n_pages, G, page_rows, d, kind, dtype), "table": table, "len": torch.tensor([150 + 30 * b, 9], dtype=torch.int32, device="cuda"),
             "new": torch.zeros(2 * n_q, 2, G, d, dtype=dtype, device="cuda"), "q": torch.zeros(2 * n_q, H, d, dtype=dtype, device="cuda"),
             "stream": torch.cuda.Stream(), "graph": torch.cuda.CUDAGraph(), "seqs": [mvla.Seq(q_row=0, n_q=n_q, n_kv=most), mvla.Seq(q_row=n_q, n_q=n_q, n_kv=most)]}

        def step(r=r):
            r["len"] += n_q
            ctx.page_write(r["pool"], r["seqs"], r["table"], r["new"][:, 0], r["new"][:, 1], kv_len=r["len"])
            return ctx.page_attention(r["pool"], r["seqs"], r["table"], r["q"], kv_len=r["len"])

        with torch.cuda.stream(r["stream"]):
            before = [None if t is None else t.clone() for t in (r["pool"].k, r["pool"].v, r["pool"].k_scale, r["pool"].v_scale, r["len"])]
            step()
            for t, o in zip((r["pool"].k, r["pool"].v, r["pool"].k_scale, r["pool"].v_scale, r["len"]), before):
                if t is not None:
                    P.bits(t).copy_(P.bits(o))
            torch.cuda.synchronize()
            with torch.cuda.graph(r["graph"], stream=r["stream"]):
                r["out"] = step()
        runs.append(r)
    for _ in range(steps):
        for r in runs:
            r["new"].copy_(torch.randn(r["new"].shape, generator=gen, device="cuda"))
            r["q"].copy_(torch.randn(r["q"].shape, generator=gen, device="cuda"))
        torch.cuda.synchronize()
        for r in runs:
            with torch.cuda.stream(r["stream"]):
                r["graph"].replay()
        torch.cuda.synchronize()
        for r in runs:
            want = P.attention(r["pool"], kind, r["seqs"], r["table"], r["q"], page_rows, kv_len=r["len"])
            for b, (s, w) in enumerate(zip(r["seqs"], want)):
                tol = P.tolerance(w, d, dtype, kind, n_q * (H // G) <= 16)
                assert ((r["out"][s.q_row:s.q_row + n_q].double() - w["out"]).abs() <= tol).all()
                j = torch.arange(int(r["len"][b]) - n_q, int(r["len"][b]), device="cuda")
                page = r["table"][b].long()[j // page_rows]
                assert same(P.pick(r["pool"].k, page, j % page_rows).double(), P.quantise(r["new"][s.q_row:s.q_row + n_q, 0], kind)[1].double())


def test_shared_pages():
    """Sequences that begin with the same pages, and two that are the same."""
    gen = generator(15)
    H, G, d, page_rows = 8, 4, 64, 32
    ctx = context(BF16, H, G, d)
    for kind in KINDS:
        pool = P.make_pool(gen, 12, G, page_rows, d, kind, BF16)
        table = torch.tensor([[0, 1, 2, 3], [0, 1, 4, 5], [0, 1, 2, 3], [6, 6, 6, 6]], dtype=torch.int32, device="cuda")
        for n_q in (1, 30):
            seqs = [mvla.Seq(q_row=30 * b, n_q=n_q, n_kv=100 + b) for b in range(4)]
            q = torch.randn(120, H, d, generator=gen, device="cuda").to(BF16)
            check_attention(ctx, pool, kind, seqs, table, q, page_rows)


def test_on_a_stream_of_its_own():
    gen = generator(16)
    H, G, d = 8, 4, 128
    ctx = context(BF16, H, G, d)
    table, pool = some_pages(ctx, gen, E4M3, G, d, 64, [900])
    q = torch.randn(40, H, d, generator=gen, device="cuda").to(BF16)
    seqs = [mvla.Seq(n_q=40, n_kv=900)]
    want = ctx.page_attention(pool, seqs, table, q)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    got = ctx.page_attention(pool, seqs, table, q, stream=st)
    k, _ = ctx.page_read(pool, seqs, table, stream=st)
    st.synchronize()
    assert torch.equal(got, want) and same(k.double(), P.rows_of(pool, E4M3, table, 0, 900, 64)[0][860:])


def test_what_the_binding_refuses():
    gen = generator(17)
    H, G, d, n = 8, 4, 64, 40
    ctx = context(BF16, H, G, d)
    seqs = [mvla.Seq(n_q=4, n_kv=n)]
    table, pool = some_pages(ctx, gen, E4M3, G, d, 16, [n])
    q = torch.zeros(4, H, d, dtype=BF16, device="cuda")
    new = torch.zeros(4, G, d, dtype=BF16, device="cuda")

    def refused(call, *what):
        with pytest.raises(what or AssertionError):
            call()

    def pools(**kw):
        return mvla.PagePool(**{**dict(k=pool.k, v=pool.v, k_scale=pool.k_scale, v_scale=pool.v_scale), **kw})

    bad = [pools(k=None), pools(k=pool.k.float()), pools(v=pool.v[:-1]), pools(k=pool.k[..., :32].contiguous(), v=pool.v[..., :32].contiguous()), pools(k_scale=None),
           pools(k_scale=None, v_scale=None), pools(k_scale=pool.k_scale[:-1]), pools(k_scale=pool.k_scale.int()), pools(k=pool.k.transpose(1, 2)), pools(k=pool.k.cpu()),
           pools(k=P.bits(pool.k), v=P.bits(pool.v)), pools(k=pool.k[0], v=pool.v[0]), mvla.PagePool(torch.zeros(4, G, 16, d, device="cuda"), torch.zeros(4, G, 16, d, device="cuda"))]
    for p in bad:
        refused(lambda: ctx.page_attention(p, seqs, table, q))
        refused(lambda: ctx.page_write(p, seqs, table, new, new))
        refused(lambda: ctx.page_read(p, seqs, table))
    for t in (table.long(), table[0], table.cpu(), torch.cat([table, table]), None):
        refused(lambda: ctx.page_attention(pool, seqs, t, q))
        refused(lambda: ctx.page_write(pool, seqs, t, new, new))
    refused(lambda: ctx.page_attention(pool, seqs, table, q.float()))
    refused(lambda: ctx.page_attention(pool, seqs, table, q[:, :4].contiguous()))
    refused(lambda: ctx.page_attention(pool, seqs, table, q, window=0))
    refused(lambda: ctx.page_attention(pool, seqs, table, q, n_sink=-1))
    refused(lambda: ctx.page_attention(pool, seqs, table, q, lse=torch.zeros(4, H + 1, device="cuda")))
    refused(lambda: ctx.page_attention(pool, seqs, table, q, kv_len=torch.zeros(2, dtype=torch.int32, device="cuda")))
    refused(lambda: ctx.page_write(pool, seqs, table, None, None))
    refused(lambda: ctx.page_write(pool, seqs, table, new[:3], new))
    refused(lambda: ctx.page_write(pool, seqs, table, new.float(), new.float()))
    E = mvla.MvlaError
    refused(lambda: ctx.page_attention(pool, [mvla.Seq(n_q=5, n_kv=n)], table, q), E)
    refused(lambda: ctx.page_attention(pool, [mvla.Seq(n_q=4, n_kv=49)], table, q), E)
    refused(lambda: ctx.page_attention(pool, seqs, table, q, out=q), E)
    refused(lambda: ctx.page_attention(pool, seqs, table, q, scale=-1.0), E)
    refused(lambda: ctx.page_attention(pool, [mvla.Seq()] * 9, torch.zeros(9, 3, dtype=torch.int32, device="cuda"), q), E)
    refused(lambda: ctx.page_write(pool, [mvla.Seq(q_row=1, n_q=4, n_kv=n)], table, new, new), E)
    refused(lambda: ctx.page_read(pool, [mvla.Seq(n_q=3, n_kv=n)] * 2, torch.cat([table, table]), k_out=new), E)
    odd = mvla.PagePool(torch.zeros(4, G, 24, d, dtype=BF16, device="cuda"), torch.zeros(4, G, 24, d, dtype=BF16, device="cuda"))
    refused(lambda: ctx.page_attention(odd, seqs, table, q), E)
    fp32 = context(FP32, H, G, d)
    refused(lambda: fp32.page_attention(pool, seqs, table, q))
    fp8 = context(FP8, H, G, d)                                # rows beside an e4m3 context's cache are bf16
    assert torch.equal(fp8.page_attention(pool, seqs, table, q), ctx.page_attention(pool, seqs, table, q))
