"""Attention over a cache in pages in 64 bits, with a tolerance that is made for every query of its own: of the rows that it sees, by the weight that it gives them."""
import torch

import page_util as P
import serve_util as U
from page_util import E2M1, E4M3, ROWS
from paper_2604_09244_b200 import mvla


def reference(pool, kind, s, table, b, q, page_rows, fp16, window=None, n_sink=0, scale=0.0, n=None):
    """dict of out, tol [n_q, H, d], lse, lse_tol [n_q, H], rows (those that see something).  `fp16`: the type in which weights meet the values, else bf16.

    A score is off by e_j: a dot product of d terms in 32 bits in any order, sums perhaps cut off ((2 d + 16) 2^-24 of the sum of magnitudes); queries as fp16, the
    largest element between 2^14 and 2^15, those below 2^-14 (2^-28 of the largest at least) off by 2^-25 (2^-39); e2m1 groups below 2^-27 of the row's largest scale: nothing instead of
    6 2^-28 of it, with a largest element of 3 times it at least; the difference to a reference (2^-23 of score and reference, in powers of two).  exp(e_j) - 1 of a weight then, in the
    numerator and, averaged by the weights, in the denominator; or, where one row's score decides, by what the others' weights can be beside it: exp(l_j + e_j - l + e) of that one's l and e; fp16: the reference with the
    exponents of scales, 2^-24 of 1024 and 256 at most, from which a tile's weights are taken; 2^-20 for the powers of two, 2 keys 2^-24 for sums and rescalings, half a step of the type in
    which the weight meets the values.  fp16: a weight times scale is counted in units of 2^-7 of the largest such product so far (2^-8 of which may be the reference): where no
    normal number is left it is off by 2^-25 2^-7 of the largest product, times a code, whose row's largest is half of the largest code at least: 2^-31 of the
    largest weight times largest element; a weight below 2^-126 of its reference is
    nothing in 32 bits, and what was summed up is, where the reference rises by as much: at most 2^8 (a reference may lie so far below a weight) times 2^-126 of a value.  e2m1 values below 2^-27 of their row's largest scale: as above.  Then the rounding of the result."""
    H, d = q.shape[1], q.shape[2]
    n = s.n_kv if n is None else n
    k, v = P.rows_of(pool, kind, table, b, n, page_rows)
    G = k.shape[1]
    c, p = torch.arange(n, device=q.device), torch.arange(s.n_q, device=q.device) + (n - s.n_q)
    sees = c[None] <= p[:, None]
    if window is not None:
        sees = sees & ((p[:, None] - c[None] < window) | (c[None] < n_sink))
    used = sees.any(0)
    k, v = (torch.where(used[:, None, None], x, 0.0).repeat_interleave(H // G, 1) for x in (k, v))
    x = q[s.q_row:s.q_row + s.n_q].double()
    scale = scale or d ** -0.5
    l = torch.einsum("ihd,jhd->hij", x, k) * scale
    e = (2 * d + 16) * 2.0 ** -24 * torch.einsum("ihd,jhd->hij", x.abs(), k.abs()) * scale
    k_top, v_top = k.abs().amax(-1).T, v.abs().amax(-1).T                       # [H, n]
    if kind != ROWS:
        most = x.abs().amax(-1, keepdim=True)
        e += torch.einsum("ihd,jhd->hij", torch.where((x != 0) & (x.abs() < 2.0 ** -28 * most), 2.0 ** -39 * most, 0.0), k.abs()) * scale
    if kind == E2M1:
        e += torch.einsum("ihd,jhd->hij", x.abs(), torch.minimum(k.abs(), 2.0 ** -27 * k_top.T[..., None])) * scale
    some = sees.any(1)
    l = l.masked_fill(~sees[None], float("-inf"))
    top = torch.where(some, l.amax(-1), 0.0) if n else torch.zeros(H, s.n_q, device=q.device, dtype=torch.float64)
    e = e + 2.0 ** -22 + 2.0 ** -23 * (torch.where(sees[None], l.abs(), 0.0) + top.abs()[..., None])
    lse = torch.logsumexp(l, -1) if n else torch.full((H, s.n_q), float("-inf"), device=q.device, dtype=torch.float64)
    w = torch.exp(l - torch.where(some[None], lse, 0.0)[..., None])
    off = torch.exp((l - torch.where(some[None], lse, 0.0)[..., None] + e).clamp(max=700.0)) - w
    keys = int(sees.sum(1).max()) if n and s.n_q else 0
    out = torch.einsum("hij,jhd->ihd", w, v)
    weight = torch.einsum("hij,jhd->ihd", w, v.abs())
    below = off.sum(-1).T[..., None]                                            # [n_q, H, 1]
    meet = U.HALF[torch.float16 if fp16 else torch.bfloat16] if q.dtype != torch.float32 else 0.0
    own = torch.einsum("hij,jhd->ihd", off, v.abs()) + below * weight
    if n:
        first = l.argmax(-1, keepdim=True)
        beside = torch.exp((l + e - (l - e).gather(-1, first)).clamp(max=0.0)).scatter(-1, first, 0.0).nan_to_num(0.0)
        beside = beside.scatter(-1, first, beside.sum(-1, keepdim=True).clamp(max=1.0))
        own = torch.minimum(own, torch.einsum("hij,jhd->ihd", beside, v.abs()))
        below = torch.minimum(below, (e.gather(-1, first) + beside.gather(-1, first))[..., 0].T[..., None])
    if fp16 and kind != ROWS:
        own = own + 2.0 ** -24 * (1.5 * top.T.abs().clamp(max=1024.0) + 256)[..., None] * weight
    own = own + (2.0 ** -20 + 2 * keys * 2.0 ** -24 + meet) * weight
    if kind != ROWS and fp16:
        product = w * v_top[:, None]
        own = own + keys * 2.0 ** -31 * (product.amax(-1) if n else w.sum(-1)).T[..., None]
        if kind == E2M1:
            own = own + torch.einsum("hij,jhd->ihd", w, torch.minimum(v.abs(), 2.0 ** -27 * v_top.T[..., None]))
    own = own + 2.0 ** -118 * torch.einsum("ij,jhd->ihd", sees.double(), v.abs())
    half = U.HALF[q.dtype]
    return {"out": out, "tol": own + half * (out.abs() + own) + 2.0 ** -134, "lse": lse.T, "rows": some,
            "lse_tol": below[..., 0] + 2.0 ** -18 + 2.0 ** -22 * torch.where(some[:, None], lse.T.abs(), 0.0)}


def check(ctx, pool, kind, seqs, table, q, page_rows, fp16, **kw):
    lse = torch.full(q.shape[:2], 77.0, device="cuda")
    out = ctx.page_attention(pool, seqs, table, q, lse=lse, **kw)
    torch.cuda.synchronize()
    for b, s in enumerate(seqs):
        r = reference(pool, kind, s, table, b, q, page_rows, fp16, **kw)
        at = slice(s.q_row, s.q_row + s.n_q)
        got, z, rows = out[at].double(), lse[at].double(), r["rows"]
        assert got.isfinite().all() and (got[~rows] == 0).all() and (z[~rows] == float("-inf")).all()
        bad = (got - r["out"]).abs() - r["tol"]
        assert (bad <= 0).all(), f"off by {(bad / r['tol']).max() + 1} tolerances in {int((bad > 0).sum())} of {bad.numel()}"
        assert ((z - r["lse"]).abs()[rows] <= r["lse_tol"][rows]).all(), f"lse off by {((z - r['lse']).abs() - r['lse_tol'])[rows].max()}"
    return out
