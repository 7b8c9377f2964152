"""The calls around the prune point (norms and rotation, windowed attention, cache eviction) against 64-bit references."""
import ctypes as C

import pytest
import torch

import serve_util as R
from paper_2604_09244_b200 import mvla
from paper_2604_09244_b200.mvla import Seq

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32, "fp8": torch.float8_e4m3fn}


def context(dtype, H, G, d, batch=8):
    return mvla.PruneContext(dtype=TYPES[dtype], n_heads=H, head_dim=d, d_model=H * d, max_batch=batch, max_text=16, max_2d=16, max_3d=16,
                             n_kv_heads=G)


def randn(gen, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=gen, device="cuda") * scale).clamp(-440, 440).to(dtype)


def bits(x):
    return x.view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[x.element_size()])


# ---------------------------------------------------------------- norms and rotation
ROPE = [
    # dtype, H, G, d, rows, rot, interleaved, norm, far
    ("bf16", 4, 4, 128, 1, 128, False, True, 100),
    ("bf16", 32, 8, 128, 33, 128, False, True, 1000000),
    ("bf16", 3, 1, 96, 17, 96, True, True, 5000),
    ("bf16", 12, 4, 64, 40, 32, False, True, 5000),
    ("bf16", 2, 2, 256, 5, 256, True, False, 5000),
    ("bf16", 5, 5, 160, 9, 80, False, True, 5000),
    ("fp32", 8, 8, 64, 21, 64, False, True, 2000000000),
    ("fp32", 7, 7, 224, 3, 112, False, True, 5000),
    ("fp32", 1, 1, 192, 2, 192, True, False, 5000),
    ("fp8", 16, 2, 128, 50, 64, True, True, 1000000),
    ("fp8", 4, 4, 96, 11, 96, False, True, 5000),
    ("bf16", 4, 4, 128, 7, 0, False, True, 0),
    ("bf16", 32, 32, 128, 1000, 128, False, True, 5000),
]


@pytest.mark.parametrize("dtype,H,G,d,rows,rot,inter,norm,far", ROPE)
def test_norm_and_rotation(dtype, H, G, d, rows, rot, inter, norm, far):
    gen = torch.Generator("cuda").manual_seed(rows * 1000 + d)
    kept, wide = TYPES[dtype], R.WIDE[TYPES[dtype]]
    qkv = randn(gen, rows, (H + 2 * G) * d, dtype=wide, scale=3.0)
    q, k, v = (x.unflatten(1, (-1, d)) for x in qkv.split([H * d, G * d, G * d], 1))
    wq, wk = (randn(gen, d, dtype=wide) for _ in range(2)) if norm else (None, None)
    pos = torch.randint(0, far + 1, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    if rows > 2:
        pos[0], pos[1] = 0, far
    freq = 10000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot) if rot else None
    cache = rows + 5
    to = torch.randperm(cache, generator=gen, device="cuda")[:rows].to(torch.int32)
    kc, vc = randn(gen, cache, G, d, dtype=kept), randn(gen, cache, G, d, dtype=kept)
    k0, v0 = kc.clone(), vc.clone()
    drop = rows > 4
    if drop:
        to[2], to[3] = -1, cache                     # rows of no cache
    ctx = context(dtype, H, G, d)
    qo, ko, vo = ctx.qk_norm_rope(q, k, pos if rot else None, freq, v=v, q_weight=wq, k_weight=wk, norm=norm, eps=1e-5, interleaved=inter,
                                  k_out=kc, v_out=vc, out_rows=to)
    assert ko is kc and vo is vc and qo.dtype == kept
    zq, sq = R.rope(q, pos, freq, wq, norm, 1e-5, inter)
    zk, sk = R.rope(k, pos, freq, wk, norm, 1e-5, inter)
    if dtype == "fp8":
        zq, zk = zq.clamp(-448, 448), zk.clamp(-448, 448)
    assert bool(((qo.double() - zq).abs() <= R.rope_tolerance(zq, sq, kept, far)).all())
    live = torch.tensor([i for i in range(rows) if not (drop and i in (2, 3))], device="cuda")
    at = to[live].long()
    assert bool(((kc.double()[at] - zk[live]).abs() <= R.rope_tolerance(zk[live], sk[live], kept, far)).all())
    want_v = v[live].float().clamp(-448, 448).to(kept) if dtype == "fp8" else v[live].to(kept)
    assert torch.equal(bits(vc)[at], bits(want_v.contiguous()))
    other = torch.ones(cache, dtype=torch.bool, device="cuda")
    other[at] = False
    assert torch.equal(bits(kc)[other], bits(k0)[other]) and torch.equal(bits(vc)[other], bits(v0)[other])
    # packed outputs of the call's own, and q alone: the same rows
    qo2, ko2, vo2 = ctx.qk_norm_rope(q, k, pos if rot else None, freq, v=v, q_weight=wq, k_weight=wk, norm=norm, eps=1e-5, interleaved=inter)
    assert torch.equal(bits(qo2), bits(qo)) and torch.equal(bits(ko2)[live], bits(kc)[at]) and torch.equal(bits(vo2)[live], bits(vc)[at])
    qo3, none, _ = ctx.qk_norm_rope(q, None, pos if rot else None, freq, q_weight=wq, norm=norm, eps=1e-5, interleaved=inter)
    assert none is None and torch.equal(bits(qo3), bits(qo))
    if dtype != "fp8":                               # in place
        x, y = q.contiguous(), k.contiguous()
        ctx.qk_norm_rope(x, y, pos if rot else None, freq, q_weight=wq, k_weight=wk, norm=norm, eps=1e-5, interleaved=inter, q_out=x, k_out=y)
        assert torch.equal(bits(x), bits(qo)) and torch.equal(bits(y), bits(ko2))
    ctx.close()


def test_rotation_of_no_rows_and_refusals():
    ctx = context("bf16", 4, 2, 64)
    q = torch.randn(6, 4, 64, device="cuda").bfloat16()
    k = torch.randn(6, 2, 64, device="cuda").bfloat16()
    pos = torch.arange(6, device="cuda", dtype=torch.int32)
    freq = torch.ones(16, device="cuda", dtype=torch.float64)
    qo, ko, _ = ctx.qk_norm_rope(q[:0], k[:0], pos[:0], freq)
    assert qo.shape == (0, 4, 64) and ko.shape == (0, 2, 64)
    with pytest.raises(mvla.MvlaError):
        ctx.qk_norm_rope(q, k, pos, freq[:15])                       # 30 elements: no multiple of 16
    with pytest.raises(mvla.MvlaError):
        ctx.qk_norm_rope(q, k, pos, torch.ones(40, device="cuda", dtype=torch.float64))
    with pytest.raises(mvla.MvlaError):
        ctx.qk_norm_rope(q, k, None, freq)
    with pytest.raises(mvla.MvlaError):
        ctx.qk_norm_rope(q, k, pos, freq, q_weight=torch.ones(64, device="cuda").bfloat16(), norm=False)
    with pytest.raises(mvla.MvlaError):
        ctx.qk_norm_rope(q[:5], None, pos[:5], freq, q_out=q[1:])    # overlaps, and is not the same rows
    for bad in (q.float(), q[:, :2], q.transpose(1, 2)):
        with pytest.raises(AssertionError):
            ctx.qk_norm_rope(bad, k, pos, freq)
    with pytest.raises(AssertionError):
        ctx.qk_norm_rope(q, k, pos.long(), freq)
    with pytest.raises(AssertionError):
        ctx.qk_norm_rope(q, k, pos[:5], freq)
    ctx.close()


# ---------------------------------------------------------------- windowed attention
def kv_layout(lens, gap=3):
    rows, at = [], 0
    for n in lens:
        rows.append(at)
        at += n + gap
    return rows, at


def attend_case(dtype, H, G, d, nq, nkv, window=None, n_sink=0, pos="count", seed=0, mass=True, lens=None, scale=0.0):
    """Random inputs of such a call; cache rows that nobody may look at hold NaN."""
    gen = torch.Generator("cuda").manual_seed(seed * 7919 + sum(nq) + 31 * sum(nkv))
    kept = TYPES[dtype]
    q_rows, q_all = kv_layout(nq, 1)
    kv_rows, kv_all = kv_layout(nkv)
    seqs = [Seq(q_row=a, n_q=b, kv_row=c, n_kv=e) for a, b, c, e in zip(q_rows, nq, kv_rows, nkv)]
    q, k, v = (randn(gen, n, h, d) for n, h in ((q_all, H), (kv_all, G), (kv_all, G)))
    k = torch.where(torch.rand(kv_all, 1, 1, generator=gen, device="cuda") < 0.1, k * 3, k)
    q_pos = kv_pos = None
    if pos != "count":
        q_pos = torch.full((q_all,), -1, dtype=torch.int32, device="cuda")
        kv_pos = torch.full((kv_all,), -1, dtype=torch.int32, device="cuda")
        for s in seqs:
            p = torch.randperm(2 * s.n_kv + 4, generator=gen, device="cuda")[:s.n_kv].sort().values.to(torch.int32)
            q_pos[s.q_row:s.q_row + s.n_q] = p[s.n_kv - s.n_q:]
            if pos == "filled":
                p = p[torch.randperm(s.n_kv, generator=gen, device="cuda")]
                p[torch.rand(s.n_kv, generator=gen, device="cuda") < 0.1] = -1          # rows that nobody sees
            kv_pos[s.kv_row:s.kv_row + s.n_kv] = p
    dead = torch.ones(kv_all, dtype=torch.bool, device="cuda")
    for b, s in enumerate(seqs):
        dead[s.kv_row:s.kv_row + (s.n_kv if lens is None else max(0, min(lens[b], s.n_kv)))] = False
    if kv_pos is not None:
        dead |= kv_pos < 0
    k[dead], v[dead] = float("nan"), float("nan")
    kv_len = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    return dict(seqs=seqs, q=q.to(kept), k=k.to(kept), v=v.to(kept), window=window, n_sink=n_sink, q_pos=q_pos, kv_pos=kv_pos, kv_len=kv_len,
                scale=scale), (torch.rand(kv_all, generator=gen, device="cuda") if mass else None), kept


def check_attention(ctx, args, mass, kept, stream=None):
    q, d, H = args["q"], args["q"].shape[2], args["q"].shape[1]
    out = torch.full(q.shape, 7.0, device="cuda", dtype=R.WIDE[kept])
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    before = None if mass is None else mass.clone()
    torch.cuda.synchronize()
    got = ctx.window_attention(**args, out=out, lse=lse, mass=mass, stream=stream)
    assert got is out
    torch.cuda.synchronize()
    refs = R.attention(**args)
    q_free = torch.ones(q.shape[0], dtype=torch.bool, device="cuda")
    kv_free = torch.ones(args["k"].shape[0], dtype=torch.bool, device="cuda")
    for s, r in zip(args["seqs"], refs):
        rows = slice(s.q_row, s.q_row + s.n_q)
        q_free[rows] = False
        o, z = out[rows].double(), lse[rows].double()
        err, tol = (o - r["out"]).abs(), R.attention_tolerance(r, d, kept)
        assert bool((err <= tol).all()), (s, float((err / tol).max()))
        none = ~r["rows"]
        assert bool((out[rows][none] == 0).all()) and bool((z[none] == float("-inf")).all())
        zerr = (z - r["lse"])[~none].abs()
        ztol = (R.logit_error(r["reach"], d) + (r["keys"] + 8) * 2.0 ** -24 + 2.0 ** -21 * (1 + r["lse"].abs()))[~none]
        assert bool((zerr <= ztol).all()), (s, float((zerr / ztol).max()))
        if mass is not None:
            c = slice(s.kv_row, s.kv_row + r["n"])
            kv_free[c] = False
            if s.n_q:
                merr = (mass[c].double() - before[c].double() - r["mass"]).abs()
                mtol = R.mass_tolerance(r, d, s.n_q, H, before[c].double())
                assert bool((merr <= mtol).all()), (s, float((merr / mtol).max()))
    assert bool((out[q_free] == 7).all()) and bool((lse[q_free] == 7).all())
    if mass is not None:
        assert torch.equal(mass[kv_free], before[kv_free])
    # the same again, bit for bit
    out2, lse2 = torch.empty_like(out), torch.empty_like(lse)
    mass2 = None if mass is None else before.clone()
    torch.cuda.synchronize()
    ctx.window_attention(**args, out=out2, lse=lse2, mass=mass2, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(out2[~q_free], out[~q_free]) and torch.equal(lse2[~q_free], lse[~q_free])
    assert mass is None or torch.equal(mass, mass2)


HEADS = [(4, 4, 128), (8, 2, 64), (3, 3, 96), (6, 2, 160), (2, 1, 256), (7, 1, 128), (4, 2, 192), (2, 2, 224)]
TOKENS = [   # n_q, n_kv, window, sinks
    ([1], [1], None, 0),
    ([1, 1, 1], [1, 300, 77], None, 0),
    ([1, 1], [64, 65], 17, 2),
    ([1, 1, 1, 1], [700, 129, 2, 1500], 128, 4),
    ([2, 1, 0, 3], [5, 190, 40, 260], 33, 1),
]
BLOCKS = [
    ([64], [64], None, 0),
    ([129, 1, 37], [129, 1, 37], 50, 3),
    ([300], [300], 1, 0),
    ([17, 200], [400, 260], 64, 8),
    ([5, 0, 130], [3, 50, 128], None, 0),        # more queries than cached rows: the first ones see nothing
    ([260], [1100], 300, 700),
]


@pytest.mark.parametrize("pos", ["count", "filled"])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32", "fp8"])
def test_attention_of_single_tokens(dtype, heads, pos):
    ctx = context(dtype, *heads)
    for i, (nq, nkv, window, sinks) in enumerate(TOKENS):
        args, mass, kept = attend_case(dtype, *heads, nq, nkv, window, sinks, pos, seed=i, mass=i % 2 == 0)
        check_attention(ctx, args, mass, kept)
    ctx.close()


@pytest.mark.parametrize("pos", ["count", "kept", "filled"])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32", "fp8"])
def test_attention_of_blocks(dtype, heads, pos):
    ctx = context(dtype, *heads)
    for i, (nq, nkv, window, sinks) in enumerate(BLOCKS):
        if pos != "count" and any(a > b for a, b in zip(nq, nkv)):
            continue
        args, mass, kept = attend_case(dtype, *heads, nq, nkv, window, sinks, pos, seed=i, mass=i % 2 == 1)
        check_attention(ctx, args, mass, kept)
    ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp32", "fp8"])
def test_attention_lengths_on_the_device(dtype):
    ctx = context(dtype, 8, 4, 128)
    for nq, nkv, lens in (([1, 1, 1, 1], [100, 100, 300, 20], [0, 57, 999, -3]), ([9, 40, 3], [64, 500, 40], [3, 129, 40])):
        args, mass, kept = attend_case(dtype, 8, 4, 128, nq, nkv, 60, 2, "count", seed=9, lens=lens)
        check_attention(ctx, args, mass, kept)
    ctx.close()


@pytest.mark.parametrize("dtype,n_q", [("bf16", 1), ("bf16", 3), ("bf16", 40), ("bf16", 300), ("fp32", 1), ("fp32", 70), ("fp8", 1), ("fp8", 90)])
def test_attention_over_a_long_cache(dtype, n_q):
    """Long enough for the keys of one block of queries to be split."""
    ctx = context(dtype, 4, 1, 128)
    args, mass, kept = attend_case(dtype, 4, 1, 128, [n_q], [20011], None, 0, "count", seed=4)
    check_attention(ctx, args, mass, kept)
    args, mass, kept = attend_case(dtype, 4, 1, 128, [n_q, 2], [9000, 5], 5000, 6, "filled", seed=5)
    check_attention(ctx, args, mass, kept)
    ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp32", "fp8"])
def test_attention_with_large_logits(dtype):
    """Logits of hundreds: the running maximum moves far, in both directions of the keys."""
    ctx = context(dtype, 4, 2, 64)
    for nq, nkv in (([1], [700]), ([200], [500])):
        args, mass, kept = attend_case(dtype, 4, 2, 64, nq, nkv, None, 0, "count", seed=6, scale=3.0)
        check_attention(ctx, args, mass, kept)
        ramp = torch.linspace(0.1, 2.0, args["k"].shape[0], device="cuda")[:, None, None]
        for r in (ramp, ramp.flip(0)):
            b = dict(args, k=(args["k"].float() * r).to(kept))
            check_attention(ctx, b, mass, kept)
    ctx.close()


def test_attention_beside_another_stream_and_in_a_graph():
    ctx = context("bf16", 8, 2, 128)
    args, mass, kept = attend_case("bf16", 8, 2, 128, [1, 1], [3000, 911], 700, 4, "count", seed=2)
    check_attention(ctx, args, mass, kept, stream=torch.cuda.Stream())
    # captured with lengths on the device: the caches grow between replays
    kv_len = torch.tensor([500, 911], dtype=torch.int32, device="cuda")
    out = torch.empty_like(args["q"])
    m = torch.zeros(args["k"].shape[0], device="cuda")
    call = dict(args, kv_len=kv_len)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.window_attention(**call, out=out, mass=m)
    for lens in ((500, 911), (1, 3), (3000, 700)):
        kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
        m.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for s, r in zip(call["seqs"], R.attention(**call)):
            o = out[s.q_row:s.q_row + s.n_q].double()
            assert bool(((o - r["out"]).abs() <= R.attention_tolerance(r, 128, kept)).all())
            c = slice(s.kv_row, s.kv_row + r["n"])
            assert bool(((m[c].double() - r["mass"]).abs() <= R.mass_tolerance(r, 128, 1, 8, m[c].double() * 0)).all())
    ctx.close()


def test_attention_refusals():
    ctx = context("bf16", 4, 2, 64, batch=2)
    q = torch.randn(10, 4, 64, device="cuda").bfloat16()
    k, v = (torch.randn(50, 2, 64, device="cuda").bfloat16() for _ in range(2))
    i32 = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
    one = [Seq(q_row=0, n_q=2, kv_row=0, n_kv=20)]

    def refused(code, seqs=one, **kw):
        args = dict(window=8, n_sink=1)
        args.update(kw)
        with pytest.raises(mvla.MvlaError) as e:
            ctx.window_attention(seqs, q, k, v, **args)
        assert e.value.code == code
    refused(mvla.ERR_CAPACITY, one * 3)
    refused(mvla.ERR_INVALID_ARG, [Seq(q_row=9, n_q=2, n_kv=5)])
    refused(mvla.ERR_INVALID_ARG, [Seq(q_row=0, n_q=2, kv_row=40, n_kv=11)])
    refused(mvla.ERR_INVALID_ARG, [Seq(q_row=-1, n_q=2, n_kv=5)])
    refused(mvla.ERR_INVALID_ARG, [Seq(n_q=2, n_kv=5), Seq(q_row=1, n_q=2, kv_row=10, n_kv=5)])          # one query of two sequences
    refused(mvla.ERR_INVALID_ARG, [Seq(n_q=2, n_kv=5), Seq(q_row=2, n_q=2, kv_row=4, n_kv=5)], mass=torch.zeros(50, device="cuda"))
    refused(mvla.ERR_INVALID_ARG, kv_pos=i32(50))                                                        # positions of rows, none of queries
    refused(mvla.ERR_INVALID_ARG, scale=-1.0)
    refused(mvla.ERR_INVALID_ARG, scale=float("nan"))
    refused(mvla.ERR_INVALID_ARG, out=q)
    # shared cache rows without accumulated weights: a common prefix
    both = [Seq(n_q=1, n_kv=30), Seq(q_row=1, n_q=1, n_kv=30)]
    o = ctx.window_attention(both, q, k, v)
    r = R.attention(both, q, k, v)
    assert all(bool(((o[b:b + 1].double() - r[b]["out"]).abs() <= R.attention_tolerance(r[b], 64, torch.bfloat16)).all()) for b in (0, 1))
    for kw in (dict(window=0), dict(n_sink=-1), dict(q_pos=i32(9)), dict(kv_len=i32(2)), dict(mass=torch.zeros(49, device="cuda")),
               dict(lse=torch.zeros(10, 3, device="cuda")), dict(out=q.float())):
        with pytest.raises(AssertionError):
            ctx.window_attention(one, q, k, v, **kw)
    # a workspace that is too small
    lib, h = mvla.lib(), ctx._h
    out, mass = torch.empty_like(q), torch.zeros(50, device="cuda")
    a = mvla.CAttention(q=q.data_ptr(), k=k.data_ptr(), v=v.data_ptr(), q_rows=10, kv_rows=50, window=mvla.WINDOW_ALL, out=out.data_ptr(),
                        mass=mass.data_ptr())
    need = C.c_int64()
    s = mvla.c_seqs(one)
    assert lib.mvla_window_attention_workspace(h, 1, s, C.byref(a), C.byref(need)) == mvla.OK and need.value > 0
    assert lib.mvla_window_attention(h, 1, s, C.byref(a), None) == mvla.ERR_INVALID_ARG
    ctx.close()


# ---------------------------------------------------------------- eviction
def evict_case(dtype, G, d, lens, budgets, seed=0, hidden=0.0, ties=False):
    gen = torch.Generator("cuda").manual_seed(seed)
    rows, total = kv_layout(lens)
    seqs = [Seq(kv_row=a, n_kv=b, budget=c) for a, b, c in zip(rows, lens, budgets)]
    k, v = randn(gen, total, G, d, dtype=TYPES[dtype]), randn(gen, total, G, d, dtype=TYPES[dtype])
    pos = torch.full((total,), -1, dtype=torch.int32, device="cuda")
    for s in seqs:
        pos[s.kv_row:s.kv_row + s.n_kv] = torch.randperm(2 * s.n_kv + 1, generator=gen, device="cuda")[:s.n_kv].to(torch.int32)
    pos[torch.rand(total, generator=gen, device="cuda") < hidden] = -1
    mass = torch.rand(total, generator=gen, device="cuda").square()
    if ties:
        mass = (mass * 5).floor() - 1                # few values, negative ones and both zeros among them
        if ties == "zeros":
            mass[::3] *= -0.0
    return seqs, k, v, pos, mass


def check_evict(ctx, seqs, k, v, pos, mass, n_sink, n_recent, kv_len=None, in_place=False, stream=None):
    k0, v0, p0, m0 = k.clone(), v.clone(), pos.clone(), mass.clone()
    kept = torch.full_like(pos, -7)
    po, mo = (pos, mass) if in_place else (torch.full_like(pos, -7), torch.full_like(mass, -7))
    new_len = torch.full((len(seqs),), -7, dtype=torch.int32, device="cuda")
    ep, em = po.clone(), mo.clone()
    torch.cuda.synchronize()
    ctx.cache_evict(seqs, k, v, pos, mass, n_sink=n_sink, n_recent=n_recent, pos_out=None if in_place else po, mass_out=None if in_place else mo,
                    kept_idx=kept, kv_len=kv_len, kv_len_out=new_len, stream=stream)
    torch.cuda.synchronize()
    want = R.evict(seqs, p0.cpu(), m0.cpu(), n_sink, n_recent, None if kv_len is None else kv_len.cpu())
    ek, ev, ei = k0.clone(), v0.clone(), torch.full_like(pos, -7)
    for b, (s, src) in enumerate(zip(seqs, want)):
        at = s.kv_row + torch.tensor(src, dtype=torch.long, device="cuda")
        m = len(src)
        rows = slice(s.kv_row, s.kv_row + m)
        bits(ek)[rows], bits(ev)[rows] = bits(k0)[at], bits(v0)[at]
        ep[rows], em[rows], ei[rows] = p0[at], m0[at], (at - s.kv_row).to(torch.int32)
        assert int(new_len[b]) == m
    assert torch.equal(kept, ei) and torch.equal(po, ep)
    assert torch.equal(bits(mo), bits(em))
    assert torch.equal(bits(k), bits(ek)) and torch.equal(bits(v), bits(ev))


EVICT = [   # lens, budgets, sinks, recent
    ([10], [9], 1, 2),
    ([1, 5, 0], [1, 4, 0], 0, 0),
    ([33, 64, 65, 1000], [32, 10, 65, 999], 2, 5),
    ([500, 3], [0, 0], 0, 0),
    ([1500, 2049, 31], [300, 2048, 100], 4, 32),
    ([5000], [4], 2, 2),
]


@pytest.mark.parametrize("dtype,G,d", [("bf16", 8, 128), ("fp32", 3, 96), ("fp8", 1, 64), ("bf16", 5, 256)])
@pytest.mark.parametrize("ties", [False, True, "zeros"])
@pytest.mark.parametrize("case", range(len(EVICT)))
def test_eviction(dtype, G, d, ties, case):
    lens, budgets, sinks, recent = EVICT[case]
    ctx = context(dtype, G, G, d)
    for hidden in (0.0, 0.3):
        check_evict(ctx, *evict_case(dtype, G, d, lens, budgets, case, hidden, ties), sinks, recent, in_place=case % 2 == 0)
    ctx.close()


def test_eviction_of_long_caches_nan_and_infinity():
    ctx = context("bf16", 1, 1, 64)
    for n, m in ((49152, 30000), (49153, 100), (120001, 60000)):
        seqs, k, v, pos, mass = evict_case("bf16", 1, 64, [n], [m], 3)
        mass[5], mass[6], mass[7], mass[8:12] = float("nan"), float("inf"), float("-inf"), float("nan")
        check_evict(ctx, seqs, k, v, pos, mass, 4, 16, in_place=n == 49153)
    ctx.close()


def test_eviction_with_more_protected_rows_than_the_budget_holds():
    """Positions that are not unique: more rows are recent than n_recent says."""
    ctx = context("bf16", 2, 2, 64)
    seqs, k, v, pos, mass = evict_case("bf16", 2, 64, [100], [10], 8)
    pos[:100] = 50
    check_evict(ctx, seqs, k, v, pos, mass, 0, 5)
    ctx.close()


def test_eviction_lengths_on_the_device_and_in_a_graph():
    ctx = context("bf16", 2, 2, 64)
    seqs, k, v, pos, mass = evict_case("bf16", 2, 64, [200, 300, 50], [100, 150, 40], 5)
    kv_len = torch.tensor([150, 400, -1], dtype=torch.int32, device="cuda")
    check_evict(ctx, seqs, k, v, pos, mass, 2, 8, kv_len=kv_len)
    kv_len = torch.tensor([100, 120, 41], dtype=torch.int32, device="cuda")
    check_evict(ctx, seqs, k, v, pos, mass, 2, 8, kv_len=kv_len, in_place=True, stream=torch.cuda.Stream())
    # captured; lengths read and written in place
    seqs, k, v, pos, mass = evict_case("bf16", 2, 64, [200, 300], [100, 150], 6)
    kv_len = torch.tensor([180, 300], dtype=torch.int32, device="cuda")
    k0, p0, m0 = k.clone(), pos.clone(), mass.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.cache_evict(seqs, k, v, pos, mass, n_sink=1, n_recent=3, kv_len=kv_len, kv_len_out=kv_len)
    want = R.evict(seqs, p0.cpu(), m0.cpu(), 1, 3, kv_len.cpu())
    graph.replay()
    torch.cuda.synchronize()
    assert kv_len.tolist() == [100, 150]
    for _ in range(2):
        for s, src in zip(seqs, want):
            at = s.kv_row + torch.tensor(src, device="cuda")
            assert torch.equal(bits(k)[s.kv_row:s.kv_row + len(src)], bits(k0)[at]) and torch.equal(pos[s.kv_row:s.kv_row + len(src)], p0[at])
        graph.replay()                               # nothing is over its budget any more
        torch.cuda.synchronize()
        assert kv_len.tolist() == [100, 150]
    ctx.close()


def test_eviction_refusals():
    ctx = context("bf16", 2, 2, 64, batch=2)
    seqs, k, v, pos, mass = evict_case("bf16", 2, 64, [20, 20], [10, 10])

    def refused(code, seqs=seqs, **kw):
        args = dict(n_sink=1, n_recent=2)
        args.update(kw)
        with pytest.raises(mvla.MvlaError) as e:
            ctx.cache_evict(seqs, k, v, pos, mass, **args)
        assert e.value.code == code
    refused(mvla.ERR_CAPACITY, list(seqs) * 2)
    refused(mvla.ERR_INVALID_ARG, n_sink=5, n_recent=6)
    refused(mvla.ERR_INVALID_ARG, [Seq(kv_row=0, n_kv=20, budget=9), Seq(kv_row=19, n_kv=5, budget=9)])
    refused(mvla.ERR_INVALID_ARG, [Seq(kv_row=40, n_kv=20, budget=9)])
    refused(mvla.ERR_INVALID_ARG, kept_idx=pos)
    with pytest.raises(AssertionError):
        ctx.cache_evict(seqs, k.float(), v, pos, mass)
    with pytest.raises(AssertionError):
        ctx.cache_evict(seqs, k, v, pos.long(), mass)
    ctx.close()
