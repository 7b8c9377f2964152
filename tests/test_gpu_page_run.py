"""A cache in pages as it is used: rows of a frame normed, rotated and written, read back where the prune point scores them, the kept rows written as caches of
their own, the prefill's attention, single tokens, and a chunk of them at once.  Every step is held against the 64-bit reference of its own inputs."""
import pytest
import torch

import page_util as P
import serve_util as R
from paper_2604_09244_b200 import mvla
from paper_2604_09244_b200 import workloads as W
from paper_2604_09244_b200.mvla import Seq
from parity_util import device_tensors
from test_gpu_page import check_attention, same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,G,kind,page_rows", [("bf16", 2, P.E4M3, 32), ("bf16", 0, P.E2M1, 16), ("bf16", 2, P.ROWS, 64), ("fp32", 0, P.E4M3, 16)])
def test_frame_to_tokens_over_pages(dtype, G, kind, page_rows):
    wl = W.small_workload(6, batch=2, D=512, H=8, d=64, dtype=dtype, n_txt=(9, 17), n_2d=(90, 130), n_3d=(80, 60), n_kv_heads=G)
    H, G, d = wl.n_heads, G or wl.n_heads, wl.head_dim
    ctx = mvla.context_for(wl)
    dev = device_tensors(wl)
    wide = dev["hidden"].dtype
    gen = torch.Generator("cuda").manual_seed(4)
    w = (torch.randn(wl.d_model, (H + 2 * G) * d, generator=gen, device="cuda") * wl.d_model ** -0.5).to(wide)
    freq = 10000.0 ** (-torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d)
    pool = ctx.alloc_pages(120, page_rows=page_rows, kind=kind)
    free = torch.randperm(120, generator=gen, device="cuda").to(torch.int32).tolist()

    def table(pages):
        return torch.tensor([[free.pop() for _ in range(pages)] for _ in wl.samples], dtype=torch.int32, device="cuda")

    def rows_of(hidden, pos):
        q, k, v = (x.unflatten(1, (-1, d)) for x in (hidden @ w).split([H * d, G * d, G * d], 1))
        q, k, _ = ctx.qk_norm_rope(q, k, pos, freq)
        return q, k, v                                         # (values stay a slice of the projection)

    def check_rows(tab, seqs, k, v):
        for b, s in enumerate(seqs):
            got = P.rows_of(pool, kind, tab, b, s.n_kv, page_rows)
            for x, y in zip(got, (k, v)):
                assert same(x[s.n_kv - s.n_q:], P.quantise(y[s.q_row:s.q_row + s.n_q], kind)[0])

    # the whole frames into pages; their keys back, dense, and scored
    n = [s.n_txt + s.n_2d + s.n_3d for s in wl.samples]
    first = [s.seq_off for s in wl.samples]
    whole = table(-(-max(n) // page_rows))
    pos = torch.cat([torch.arange(m, dtype=torch.int32, device="cuda") for m in n])
    q, k, v = rows_of(dev["hidden"], pos)
    seqs = [Seq(q_row=a, n_q=m, n_kv=m) for a, m in zip(first, n)]
    ctx.page_write(pool, seqs, whole, k, v)
    check_rows(whole, seqs, k, v)
    k_back, v_back = ctx.page_read(pool, seqs, whole)
    assert k_back.dtype == wide and same(k_back.double(), P.quantise(k, kind)[0]) and same(v_back.double(), P.quantise(v, kind)[0])
    o = ctx.prune_step(0, wl.samples, wl.mode, q, k_back, v_back, dev["hidden"])
    at = o.out_offsets.tolist()
    kept = o.kept_idx[:at[-1]]
    # the kept rows: caches of their own, behind them the tokens
    m = [b - a for a, b in zip(at, at[1:])]
    steps = 5
    tab = table(-(-(max(m) + 2 * steps) // page_rows))
    seqs = [Seq(q_row=a, n_q=c, n_kv=c) for a, c in zip(at, m)]
    q, k, v = rows_of(o.out_hidden[:at[-1]], kept)
    ctx.page_write(pool, seqs, tab, k, v)
    check_rows(tab, seqs, k, v)
    check_attention(ctx, pool, kind, seqs, tab, q, page_rows, window=60, n_sink=4)
    # single tokens, then as many at once
    last = [int(kept[b - 1]) for b in at[1:]]
    hidden = torch.randn(2, 2 * steps, wl.d_model, generator=gen, device="cuda").to(wide)
    for i in range(steps):
        pos = torch.tensor([p + 1 + i for p in last], dtype=torch.int32, device="cuda")
        q, k, v = rows_of(hidden[:, i], pos)
        seqs = [Seq(q_row=b, n_q=1, n_kv=m[b] + i + 1) for b in range(2)]
        ctx.page_write(pool, seqs, tab, k, v)
        check_attention(ctx, pool, kind, seqs, tab, q, page_rows, window=60, n_sink=4)
    pos = torch.cat([torch.arange(p + 1 + steps, p + 1 + 2 * steps, dtype=torch.int32, device="cuda") for p in last])
    q, k, v = rows_of(hidden[:, steps:].flatten(0, 1), pos)
    seqs = [Seq(q_row=b * steps, n_q=steps, n_kv=m[b] + 2 * steps) for b in range(2)]
    ctx.page_write(pool, seqs, tab, k, v)
    check_rows(tab, seqs, k, v)
    check_attention(ctx, pool, kind, seqs, tab, q, page_rows, window=60, n_sink=4)
    # nothing that was written before has moved
    k_again, v_again = ctx.page_read(pool, [Seq(q_row=a, n_q=c, n_kv=c) for a, c in zip(first, n)], whole)
    assert torch.equal(k_again, k_back) and torch.equal(v_again, v_back)
    ctx.close()
