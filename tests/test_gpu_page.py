"""A cache in pages against its definition in 64 bits: rows in, rows out (both exact), attention."""
import pytest
import torch

import page_util as P
import serve_util as U
from page_util import E2M1, E4M3, ROWS
from paper_2604_09244_b200 import mvla

pytestmark = pytest.mark.gpu
BF16, FP32, FP8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


def context(dtype=BF16, H=8, G=4, d=64, batch=8):
    return mvla.PruneContext(dtype=dtype, n_heads=H, head_dim=d, d_model=H * d, max_batch=batch, max_text=32, max_2d=64, max_3d=64, n_kv_heads=G)


def generator(seed):
    return torch.Generator("cuda").manual_seed(seed)


def same(a, b):
    """Equal, NaN to NaN; zeros of either sign."""
    return bool(((a == b) | (a.isnan() & b.isnan())).all())


def check_attention(ctx, pool, kind, seqs, table, q, page_rows, *, kv_len=None, lse=True, **kw):
    H, d = q.shape[1], q.shape[2]
    G = pool.k.shape[1]
    got_lse = torch.full(q.shape[:2], 77.0, device="cuda") if lse else None
    out = torch.full_like(q, 55.0)
    back = ctx.page_attention(pool, seqs, table, q, kv_len=kv_len, out=out, lse=got_lse, **kw)
    assert back is out
    torch.cuda.synchronize()
    untouched = torch.ones(q.shape[0], dtype=torch.bool, device="cuda")
    most = max((s.n_q for s in seqs), default=0) * (H // G)
    for s, r in zip(seqs, P.attention(pool, kind, seqs, table, q, page_rows, kv_len=kv_len, **kw)):
        untouched[s.q_row:s.q_row + s.n_q] = False
        got = out[s.q_row:s.q_row + s.n_q].double()
        tol = P.tolerance(r, d, q.dtype, kind, most <= 16)
        assert ((got - r["out"]).abs() <= tol).all(), f"off by {((got - r['out']).abs() - tol).max()} beyond {tol.max()}"
        assert (got[~r["rows"]] == 0).all()
        if lse:
            z = got_lse[s.q_row:s.q_row + s.n_q].double()
            seen = r["rows"]
            assert (z[~seen] == float("-inf")).all()
            assert ((z - r["lse"]).abs()[seen] <= (2 * U.logit_error(r["reach"], d) + 2.0 ** -18 + 2.0 ** -22 * r["lse"].abs())[seen]).all()
    assert (out[untouched] == 55.0).all()
    assert not lse or (got_lse[untouched] == 77.0).all()
    return out


# ---- rows in and out

@pytest.mark.parametrize("kind", [ROWS, E4M3, E2M1])
@pytest.mark.parametrize("dtype,G,d,page_rows", [(BF16, 4, 64, 16), (BF16, 8, 128, 64), (FP8, 2, 96, 32), (FP32, 3, 160, 128), (BF16, 1, 256, 256), (FP32, 4, 64, 16),
                                                 (BF16, 5, 224, 16), (BF16, 2, 192, 32)])
def test_rows_written_and_read(kind, dtype, G, d, page_rows):
    gen = generator(1 + G + d)
    wide = U.WIDE[dtype]
    ctx = context(dtype, G * 2, G, d)
    seqs = [mvla.Seq(q_row=3, n_q=7, n_kv=7), mvla.Seq(q_row=10, n_q=1, n_kv=page_rows + 1), mvla.Seq(q_row=0, n_q=0, n_kv=40),
            mvla.Seq(q_row=12, n_q=2 * page_rows + 5, n_kv=3 * page_rows), mvla.Seq(q_row=11, n_q=1, n_kv=1)]
    rows = 12 + 2 * page_rows + 5 + 4
    table, n_pages = P.make_table(gen, [s.n_kv for s in seqs], page_rows)
    pool = P.make_pool(gen, n_pages, G, page_rows, d, kind, wide)
    before = [None if t is None else t.clone() for t in (pool.k, pool.v, pool.k_scale, pool.v_scale)]
    fused = (torch.randn(rows, 4 * G, d, generator=gen, device="cuda") * torch.exp(2 * torch.randn(rows, 4 * G, 1, generator=gen, device="cuda"))).to(wide)
    new = {"k": fused[:, :G].contiguous(), "v": fused[:, 2 * G:3 * G]}
    ctx.page_write(pool, seqs, table, new["k"], new["v"])
    k_out = torch.full((rows, G, d), 9.0, dtype=wide, device="cuda")
    v_out = k_out.clone()
    ctx.page_read(pool, seqs, table, k_out=k_out, v_out=v_out)
    torch.cuda.synchronize()
    for name, codes, scale, old, old_scale, back in (("k", pool.k, pool.k_scale, before[0], before[2], k_out), ("v", pool.v, pool.v_scale, before[1], before[3], v_out)):
        left = torch.ones(rows, dtype=torch.bool, device="cuda")
        for b, s in enumerate(seqs):
            if not s.n_q:
                continue
            j = torch.arange(s.n_kv - s.n_q, s.n_kv, device="cuda")
            page = table[b].long()[j // page_rows]
            value, code, byte = P.quantise(new[name][s.q_row:s.q_row + s.n_q], kind)
            assert same(P.pick(codes, page, j % page_rows).double(), code.double())
            if scale is not None:
                assert torch.equal(scale[page, :, j % page_rows], byte)
                old_scale[page, :, j % page_rows] = byte
            P.bits(old)[page, :, j % page_rows] = P.bits(codes)[page, :, j % page_rows]
            assert same(back[s.q_row:s.q_row + s.n_q].double(), value)
            left[s.q_row:s.q_row + s.n_q] = False
        assert torch.equal(P.bits(old), P.bits(codes))           # nothing else was written
        assert scale is None or torch.equal(old_scale, scale)
        assert (back[left] == 9.0).all()


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("kind", [E4M3, E2M1])
def test_values_where_rounding_can_go_wrong(kind, dtype):
    """Ties, the ends of the scales, zeros of both signs, what is not finite."""
    G, d, page_rows = 2, 64, 16
    ctx = context(dtype, 2, G, d)
    top = P.FORMAT[kind][0]
    x = torch.zeros(64, G, d, device="cuda")
    gen = generator(5)
    x[0] = torch.randn(G, d, generator=gen, device="cuda")
    x[1], x[1, :, ::2] = -0.0, 0.0
    for i in range(2, 10):                                     # halves of steps, at several scales
        x[i] = (torch.arange(d, device="cuda") - d // 2) * 0.125 * top / 8
        x[i] *= 2.0 ** (20 * i - 100)
    for i, big in enumerate([top, top * (1 + 2.0 ** -7), top / 2, top / 2 * (1 + 2.0 ** -7), 1.0, 1 - 2.0 ** -8, 3.0e38, 2.0 ** 127, 2.0 ** -100, 2.0 ** -117, 2.0 ** -126,
                             2.0 ** -130, 1e-38]):
        x[10 + i] = torch.rand(G, d, generator=gen, device="cuda") * big * 0.9
        x[10 + i, :, 5], x[10 + i, :, 40] = big, -big
    x[30, 0, 3], x[31, 1, 40], x[32, 0, 33] = float("nan"), float("inf"), float("-inf")
    x = x.to(dtype)
    seqs = [mvla.Seq(q_row=0, n_q=64, n_kv=64)]
    pool = ctx.alloc_pages(4, page_rows=page_rows, kind=kind)
    table = torch.tensor([[2, 0, 3, 1]], dtype=torch.int32, device="cuda")
    ctx.page_write(pool, seqs, table, x, x)
    k, v = ctx.page_read(pool, seqs, table)
    value, code, byte = P.quantise(x, kind)
    j = torch.arange(64, device="cuda")
    page = table[0].long()[j // page_rows]
    assert torch.equal(pool.k_scale[page, :, j % page_rows], byte)
    assert same(k.double(), value) and same(v.double(), value)
    assert torch.equal(P.bits(P.pick(pool.k, page, j % page_rows)), P.bits(code))


def test_rows_at_device_lengths_and_one_of_the_two_alone():
    gen = generator(3)
    G, d, page_rows = 4, 64, 16
    ctx = context(G=G, d=d)
    pool = P.make_pool(gen, 12, G, page_rows, d, E4M3, BF16)
    table = torch.randperm(12, generator=gen, device="cuda").to(torch.int32).view(3, 4).contiguous()
    seqs = [mvla.Seq(q_row=0, n_q=4, n_kv=64), mvla.Seq(q_row=4, n_q=5, n_kv=64), mvla.Seq(q_row=9, n_q=3, n_kv=50)]
    kv_len = torch.tensor([30, 2, 1000], dtype=torch.int32, device="cuda")                  # the second: three rows before the first one
    new = torch.randn(12, G, d, generator=gen, device="cuda").to(BF16)
    old = P.bits(pool.v).clone()
    ctx.page_write(pool, seqs, table, new, None, kv_len=kv_len)
    assert torch.equal(P.bits(pool.v), old)
    k = torch.full((12, G, d), 5.0, dtype=BF16, device="cuda")
    back, none = ctx.page_read(pool, seqs, table, k_out=k, kv_len=kv_len)
    assert back is k and none is None
    want = P.quantise(new, E4M3)[0]
    want[4:7] = 0
    assert same(k.double(), want)


@pytest.mark.parametrize("kind", [ROWS, E4M3, E2M1])
def test_rows_read_into_slices_of_one_tensor(kind):
    gen = generator(6)
    G, d, page_rows = 4, 96, 32
    ctx = context(G=G, d=d)
    table, n_pages = P.make_table(gen, [75, 20], page_rows)
    pool = P.make_pool(gen, n_pages, G, page_rows, d, kind, BF16)
    seqs = [mvla.Seq(q_row=30, n_q=75, n_kv=75), mvla.Seq(q_row=2, n_q=11, n_kv=20)]
    both = torch.full((110, 3, G, d), 7.0, dtype=BF16, device="cuda")
    k, v = ctx.page_read(pool, seqs, table, k_out=both[:, 2], v_out=both[:, 0])
    assert k.data_ptr() == both[:, 2].data_ptr() and v.data_ptr() == both.data_ptr()
    left = torch.ones(110, dtype=torch.bool, device="cuda")
    for b, s in enumerate(seqs):
        for at, want in zip((2, 0), P.rows_of(pool, kind, table, b, s.n_kv, page_rows)):
            assert same(both[s.q_row:s.q_row + s.n_q, at].double(), want[s.n_kv - s.n_q:])
        left[s.q_row:s.q_row + s.n_q] = False
    assert (both[left] == 7.0).all() and (both[:, 1] == 7.0).all()


def test_pages_outside_the_pool():
    """Written rows are dropped, read rows are zeros, attention sees rows of zeros."""
    gen = generator(4)
    G, d, page_rows = 4, 64, 16
    for kind in (ROWS, E4M3, E2M1):
        ctx = context(G=G, d=d)
        pool = P.make_pool(gen, 3, G, page_rows, d, kind, BF16)
        table = torch.tensor([[1, -1, 0], [3, 2, -0x80000000], [0x7FFFFFFF, -5, 4]], dtype=torch.int32, device="cuda")
        for n_q in (1, 37):
            seqs = [mvla.Seq(q_row=b * 40, n_q=n_q, n_kv=41) for b in range(3)]
            q = torch.randn(120, 8, d, generator=gen, device="cuda").to(BF16)
            check_attention(ctx, pool, kind, seqs, table, q, page_rows)
        k, v = ctx.page_read(pool, [mvla.Seq(q_row=b * 41, n_q=41, n_kv=41) for b in range(3)], table)
        for b in range(3):
            for got, want in zip((k, v), P.rows_of(pool, kind, table, b, 41, page_rows)):
                assert same(got[41 * b:41 * b + 41].double(), want)
        old = [P.bits(t).clone() for t in (pool.k, pool.v)]
        ctx.page_write(pool, [mvla.Seq(q_row=0, n_q=9, n_kv=41), mvla.Seq(q_row=9, n_q=2, n_kv=2)], table[2:].expand(2, 3).contiguous(), k, v)
        assert all(torch.equal(P.bits(t), o) for t, o in zip((pool.k, pool.v), old))


# ---- attention

SHAPES = [(8, 4, 64), (8, 8, 128), (16, 2, 96), (6, 2, 160), (4, 1, 256), (28, 4, 128), (2, 2, 192), (3, 3, 224)]


@pytest.mark.parametrize("kind", [ROWS, E4M3, E2M1])
@pytest.mark.parametrize("H,G,d", SHAPES)
def test_single_tokens(H, G, d, kind):
    gen = generator(H + G + d + kind)
    for page_rows, window, sinks, lengths in ((16, None, 0, [1, 15, 16, 17, 700, 3]), (64, 33, 2, [64, 65, 300, 1000]), (256, 1, 0, [5, 513]), (32, 200, 40, [3000, 31])):
        ctx = context(BF16, H, G, d)
        table, n_pages = P.make_table(gen, lengths, page_rows)
        pool = P.make_pool(gen, n_pages, G, page_rows, d, kind, BF16)
        seqs = [mvla.Seq(q_row=i + 1, n_q=1, n_kv=n) for i, n in enumerate(lengths)]
        q = torch.randn(len(lengths) + 2, H, d, generator=gen, device="cuda").to(BF16)
        check_attention(ctx, pool, kind, seqs, table, q, page_rows, window=window, n_sink=sinks)


@pytest.mark.parametrize("kind", [ROWS, E4M3, E2M1])
@pytest.mark.parametrize("H,G,d", SHAPES)
def test_chunks(H, G, d, kind):
    gen = generator(H + G + d + kind + 100)
    for page_rows, window, sinks, shapes in ((16, None, 0, [(40, 45), (0, 30), (3, 200), (130, 130)]), (128, 50, 3, [(70, 400), (1, 64)]), (64, None, 0, [(33, 20), (64, 640)])):
        ctx = context(BF16, H, G, d)
        table, n_pages = P.make_table(gen, [n for _, n in shapes], page_rows)
        pool = P.make_pool(gen, n_pages, G, page_rows, d, kind, BF16)
        row, seqs = 2, []
        for n_q, n in shapes:
            seqs.append(mvla.Seq(q_row=row, n_q=n_q, n_kv=n))
            row += n_q + 1
        q = torch.randn(row, H, d, generator=gen, device="cuda").to(BF16)
        check_attention(ctx, pool, kind, seqs, table, q, page_rows, window=window, n_sink=sinks)


@pytest.mark.parametrize("kind", [ROWS, E4M3, E2M1])
@pytest.mark.parametrize("n_q", [2, 3, 4, 5, 8, 16, 17])
def test_few_tokens(n_q, kind):
    """Two to sixteen tokens, about where the forms change; some sequences have fewer."""
    gen = generator(n_q)
    H, G, d, page_rows = 8, 4, 128, 32
    ctx = context(BF16, H, G, d)
    lengths = [n_q, 90, 1025, 17]
    table, n_pages = P.make_table(gen, lengths, page_rows)
    pool = P.make_pool(gen, n_pages, G, page_rows, d, kind, BF16)
    seqs = [mvla.Seq(q_row=20 * i, n_q=max(1, n_q - i), n_kv=n) for i, n in enumerate(lengths)]
    q = torch.randn(80, H, d, generator=gen, device="cuda").to(BF16)
    check_attention(ctx, pool, kind, seqs, table, q, page_rows)


@pytest.mark.parametrize("kind", [ROWS, E4M3, E2M1])
@pytest.mark.parametrize("n_q,page_rows,window", [(1, 16, None), (70, 32, None), (9, 64, 20), (200, 16, 64)])
def test_fp32(kind, n_q, page_rows, window):
    gen = generator(n_q + kind)
    ctx = context(FP32, 8, 4, 64)
    lengths = [n_q, 300]
    table, n_pages = P.make_table(gen, lengths, page_rows)
    pool = P.make_pool(gen, n_pages, 4, page_rows, 64, kind, FP32)
    seqs = [mvla.Seq(q_row=0, n_q=n_q, n_kv=n_q), mvla.Seq(q_row=n_q, n_q=n_q, n_kv=300)]
    q = torch.randn(2 * n_q, 8, 64, generator=gen, device="cuda")
    check_attention(ctx, pool, kind, seqs, table, q, page_rows, window=window, n_sink=1)


@pytest.mark.parametrize("kind", [ROWS, E4M3, E2M1])
@pytest.mark.parametrize("n_q", [1, 5, 60])
def test_rows_that_nobody_sees_may_hold_anything(kind, n_q):
    """Behind the length, outside the window, on pages of others: NaN, infinity, every byte."""
    gen = generator(17 + n_q)
    G, d, page_rows = 4, 128, 64
    ctx = context(BF16, 8, G, d)
    n, window = 1000, 100
    table, n_pages = P.make_table(gen, [n], page_rows)
    pool = P.make_pool(gen, n_pages, G, page_rows, d, kind, BF16)
    clean = [None if t is None else t.clone() for t in (pool.k, pool.v, pool.k_scale, pool.v_scale)]
    seen = torch.zeros(n_pages, page_rows, dtype=torch.bool, device="cuda")
    j = torch.arange(n - n_q - window + 1, n, device="cuda")
    seen[table[0].long()[j // page_rows], j % page_rows] = True
    seen[table[0, 0], :2] = True                               # two sinks
    for t in (pool.k, pool.v):
        junk = torch.full_like(P.bits(t), 0x7F)
        junk.random_(0, 256, generator=gen)
        junk[..., ::3] = 0xFF
        b = P.bits(t)
        b.copy_(torch.where(seen[:, None, :, None], b, junk))
    for t in (pool.k_scale, pool.v_scale):
        if t is not None:
            s = seen[:, None, :].expand(t.shape[:3])
            t.copy_(torch.where(s if t.dim() == 3 else s[..., None], t, torch.full_like(t, 255)))
    q = torch.randn(n_q, 8, d, generator=gen, device="cuda").to(BF16)
    seqs = [mvla.Seq(q_row=0, n_q=n_q, n_kv=n)]
    got = ctx.page_attention(pool, seqs, table, q, window=window, n_sink=2)
    want = ctx.page_attention(mvla.PagePool(*clean), seqs, table, q, window=window, n_sink=2)
    assert torch.isfinite(got).all() and torch.equal(got, want)


@pytest.mark.parametrize("kind", [ROWS, E4M3])
@pytest.mark.parametrize("H,G,d,page_rows,seqs,window,n_sink", [
    (8, 8, 64, 16, [(1, 1), (1, 17), (1, 4000)], None, 0),                  # cut into parts, more of them than the short ones have rows
    (6, 2, 96, 32, [(3, 900), (0, 5), (5, 40)], None, 0),                   # rows of two queries in a block
    (16, 2, 128, 64, [(1, 700), (2, 130)], 100, 5),
    (4, 4, 160, 256, [(33, 33), (7, 300)], 31, 0),
    (8, 4, 192, 128, [(2, 0), (5, 3), (9, 500)], None, 0),                  # more rows than are cached: those before row 0 see nothing
    (7, 7, 224, 16, [(20, 2000)], 1, 40),
    (8, 1, 256, 64, [(5, 1000), (1, 63)], 640, 64),
])
def test_fp32_blocks(kind, H, G, d, page_rows, seqs, window, n_sink):
    """Blocks of 8 query rows, warps with a granule of 16 keys each and without, every size of heads."""
    gen = generator(d + kind)
    ctx = context(FP32, H, G, d)
    lengths = [n for _, n in seqs]
    table, n_pages = P.make_table(gen, lengths, page_rows)
    pool = P.make_pool(gen, n_pages, G, page_rows, d, kind, FP32)
    rows = [0]
    for n_q, _ in seqs:
        rows.append(rows[-1] + n_q + 1)
    q = torch.randn(rows[-1], H, d, generator=gen, device="cuda")
    seqs = [mvla.Seq(q_row=r, n_q=n_q, n_kv=n) for r, (n_q, n) in zip(rows, seqs)]
    check_attention(ctx, pool, kind, seqs, table, q, page_rows, window=window, n_sink=n_sink)


@pytest.mark.parametrize("n_q", [1, 3, 40])
def test_fp32_rows_that_nobody_sees_may_hold_anything(n_q):
    gen = generator(40 + n_q)
    G, d, page_rows, n, window = 4, 64, 32, 1500, 90
    ctx = context(FP32, 8, G, d)
    table, n_pages = P.make_table(gen, [n], page_rows)
    pool = P.make_pool(gen, n_pages, G, page_rows, d, ROWS, FP32)
    clean = mvla.PagePool(pool.k.clone(), pool.v.clone())
    seen = torch.zeros(n_pages, page_rows, dtype=torch.bool, device="cuda")
    j = torch.arange(n - 9 - n_q - window + 1, n - 9, device="cuda")         # (nine rows of the descriptor's are not there yet)
    seen[table[0].long()[j // page_rows], j % page_rows] = True
    seen[table[0, 0], :3] = True
    for t in (pool.k, pool.v):
        t.masked_fill_(~seen[:, None, :, None], float("nan"))
    q = torch.randn(n_q, 8, d, generator=gen, device="cuda")
    seqs = [mvla.Seq(q_row=0, n_q=n_q, n_kv=n)]
    kv_len = torch.tensor([n - 9], dtype=torch.int32, device="cuda")
    got = ctx.page_attention(pool, seqs, table, q, window=window, n_sink=3, kv_len=kv_len)
    want = ctx.page_attention(clean, seqs, table, q, window=window, n_sink=3, kv_len=kv_len)
    assert torch.isfinite(got).all() and torch.equal(got, want)


@pytest.mark.parametrize("d", [64, 96, 128, 160, 192, 224, 256])
@pytest.mark.parametrize("H,G,n_q", [(4, 4, 1), (8, 2, 2), (6, 2, 3), (2, 1, 8), (2, 2, 16)])
def test_few_rows_of_their_own_type(d, H, G, n_q):
    """Short sequences over bf16 pages, up to 16 query rows to a key head, every size of heads; rows that see nothing."""
    gen = generator(d + n_q)
    page_rows = 16
    ctx = context(BF16, H, G, d)
    lengths = [n_q, 0, 300, 65, 1]
    table, n_pages = P.make_table(gen, lengths, page_rows)
    pool = P.make_pool(gen, n_pages, G, page_rows, d, ROWS, BF16)
    seqs = [mvla.Seq(q_row=20 * i, n_q=n_q, n_kv=n) for i, n in enumerate(lengths)]
    q = torch.randn(100, H, d, generator=gen, device="cuda").to(BF16)
    check_attention(ctx, pool, ROWS, seqs, table, q, page_rows)
    check_attention(ctx, pool, ROWS, seqs, table, q, page_rows, window=40, n_sink=2)


@pytest.mark.parametrize("kind", [E4M3, E2M1])
@pytest.mark.parametrize("H,G,d,n_q,page_rows,window,n_sink", [
    (32, 32, 64, 200, 16, None, 0), (32, 32, 96, 129, 64, None, 0), (32, 32, 128, 256, 32, 2100, 70), (96, 32, 128, 80, 128, None, 0),     # two tiles of rows that share what is unpacked
    (24, 24, 160, 140, 16, None, 0), (24, 24, 256, 256, 64, 2500, 1),                                                                     # one each
])
def test_two_blocks_over_long_sequences(kind, H, G, d, n_q, page_rows, window, n_sink):
    gen = generator(d + n_q + kind)
    ctx = context(BF16, H, G, d)
    lengths = [2900, 2777, 3000]
    table, n_pages = P.make_table(gen, lengths, page_rows)
    pool = P.make_pool(gen, n_pages, G, page_rows, d, kind, BF16)
    seqs = [mvla.Seq(q_row=0, n_q=n_q, n_kv=2900), mvla.Seq(q_row=n_q, n_q=0, n_kv=2777), mvla.Seq(q_row=n_q + 1, n_q=n_q // 2 - 3, n_kv=3000)]
    q = torch.randn(2 * n_q, H, d, generator=gen, device="cuda").to(BF16)
    check_attention(ctx, pool, kind, seqs, table, q, page_rows, window=window, n_sink=n_sink)
    kv_len = torch.tensor([2500, 5, 61], dtype=torch.int32, device="cuda")
    check_attention(ctx, pool, kind, seqs, table, q, page_rows, window=window, n_sink=n_sink, kv_len=kv_len)


@pytest.mark.parametrize("call", list(P.CLUSTERS))
def test_clusters(call):
    """Parts of a block of queries joined inside clusters of two, four and eight CTAs, and behind clusters."""
    kind, H, G, d, lengths = call
    gen = generator(d + H)
    page_rows = 64
    ctx = context(BF16, H, G, d)
    table, n_pages = P.make_table(gen, [n for _, n in lengths], page_rows)
    pool = P.make_pool(gen, n_pages, G, page_rows, d, kind, BF16)
    seqs, row = [], 0
    for n_q, n in lengths:
        seqs.append(mvla.Seq(q_row=row, n_q=n_q, n_kv=n))
        row += n_q + 1
    q = torch.randn(row, H, d, generator=gen, device="cuda").to(BF16)
    check_attention(ctx, pool, kind, seqs, table, q, page_rows)
    check_attention(ctx, pool, kind, seqs, table, q, page_rows, kv_len=torch.tensor([n // 3 for _, n in lengths], dtype=torch.int32, device="cuda"))
