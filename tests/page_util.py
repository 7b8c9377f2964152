"""A cache in pages in 64 bits, written from its definition, with how far a result may be off."""
import torch

import serve_util as U
from paper_2604_09244_b200 import mvla

ROWS, E4M3, E2M1 = mvla.PAGE_ROWS, mvla.PAGE_E4M3, mvla.PAGE_E2M1
# largest number, bits behind the point, exponent of the smallest normal number, and the largest exponent of a scale
FORMAT = {E4M3: (448.0, 3, -6, 119), E2M1: (6.0, 1, 0, 125)}


def exponents(x, kind):
    """Exponent of the scale of every group [..., groups] of rows [..., d]; 128 where something is not finite."""
    x = x.double().unflatten(-1, (-1, x.shape[-1] if kind == E4M3 else 32))
    top, _, _, most = FORMAT[kind]
    big = x.abs().amax(-1)
    fine = torch.isfinite(x).all(-1)
    m, e = torch.frexp(torch.where(fine, big, 1.0) / top)          # big / top = m 2^e, 1/2 <= m < 1 (top 2^e is exact, the quotient's order is not touched)
    e = e.long()
    e = torch.where(top * torch.exp2(e.double() - 1) >= big, e - 1, e)
    e = torch.where(top * torch.exp2(e.double()) < big, e + 1, e)
    e = torch.where(big == 0, -117, e).clamp(-117, most)
    return torch.where(fine, e, 128)


def quantise(x, kind):
    """(values, codes, scale bytes) of rows [..., d]: values in 64 bits, codes and bytes as the pool holds them."""
    if kind == ROWS:
        return x.double(), x, None
    _, bits, least, _ = FORMAT[kind]
    top = FORMAT[kind][0]
    e = exponents(x, kind)
    g = x.unflatten(-1, (-1, x.shape[-1] if kind == E4M3 else 32)).double()
    y = torch.where(e[..., None] == 128, 0.0, g / torch.exp2(e.double())[..., None])
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** least))) - bits)
    y = ((y / step).round() * step).clamp(-top, top)
    value = torch.where(e[..., None] == 128, float("nan"), y * torch.exp2(e.double())[..., None]).flatten(-2)
    y = y.flatten(-2)
    if kind == E4M3:
        return value, y.float().to(torch.float8_e4m3fn), (e.squeeze(-1) + 127).to(torch.uint8)
    steps = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=x.device)
    code = torch.searchsorted(steps, y.abs()).to(torch.uint8) | torch.signbit(y).to(torch.uint8) << 3
    return value, code[..., 0::2] | code[..., 1::2] << 4, (e + 127).to(torch.uint8)


def values(codes, scale, kind):
    """What codes and scale bytes stand for, 64 bits (bytes 1 .. 254)."""
    if kind == ROWS:
        return codes.double()
    if kind == E4M3:
        return codes.double() * torch.exp2(scale.double() - 127)[..., None]
    steps = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=codes.device)
    steps = torch.cat([steps, -steps])
    y = torch.stack([steps[(codes & 15).long()], steps[(codes >> 4).long()]], -1).flatten(-2)
    return (y.unflatten(-1, (-1, 32)) * torch.exp2(scale.double() - 127)[..., None]).flatten(-2)


def bits(t):
    return t.view(torch.uint8) if t.dtype != torch.uint8 else t


def pick(t, page, row):
    """[n, heads, ...] of a pool's tensor: rows `row` of pages `page`."""
    if t.dtype == torch.float8_e4m3fn:
        return t.view(torch.uint8)[page, :, row].view(t.dtype)
    return t[page, :, row]


def make_pool(gen, n_pages, G, P, d, kind, wide, spread=0.7, device="cuda"):
    """A pool of pages full of rows, as the definition stores them."""
    out = []
    for _ in range(2):
        x = torch.randn(n_pages, G, P, d, generator=gen, device=device) * torch.exp(torch.randn(G, 1, d, generator=gen, device=device) * spread)
        _, codes, scale = quantise(x.to(wide).float() if kind != ROWS else x.to(wide), kind)
        out.append((codes.contiguous(), scale.contiguous() if scale is not None else None))
    return mvla.PagePool(out[0][0], out[1][0], out[0][1], out[1][1])


def make_table(gen, lengths, P, spare=3, device="cuda"):
    """(table, pages of the pool) for sequences of such lengths, pages in no order; entries nobody needs are far outside."""
    need = [-(-n // P) for n in lengths]
    n_pages = sum(need) + spare
    order = torch.randperm(n_pages, generator=gen, device=device).to(torch.int32)
    table = torch.full((len(lengths), max(max(need), 1)), 0x7FFFFFFF, dtype=torch.int32, device=device)
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = order[at:at + m]
        at += m
    return table, n_pages


def rows_of(pool, kind, table, b, n, P):
    """Cached rows 0 .. n - 1 of sequence b: (k, v) [n, heads, d] in 64 bits; pages outside the pool are zeros."""
    j = torch.arange(n, device=table.device)
    page = table[b].long()[j // P]
    there = (page >= 0) & (page < pool.k.shape[0])
    page = torch.where(there, page, 0)
    out = []
    for codes, scale in ((pool.k, pool.k_scale), (pool.v, pool.v_scale)):
        x = values(pick(codes, page, j % P), None if scale is None else scale[page, :, j % P], kind)
        out.append(torch.where(there[:, None, None], x, 0.0))
    return out


def attention(pool, kind, seqs, table, q, P, window=None, n_sink=0, scale=0.0, kv_len=None):
    """As serve_util.attention, over the pages: and per sequence the largest value."""
    found = []
    for b, s in enumerate(seqs):
        n = s.n_kv if kv_len is None else max(0, min(int(kv_len[b]), s.n_kv))
        k, v = rows_of(pool, kind, table, b, n, P)
        r = U.attention([mvla.Seq(q_row=s.q_row, n_q=s.n_q, kv_row=0, n_kv=n)], q, k, v, window=window, n_sink=n_sink, scale=scale)[0]
        r["largest"] = float(v[torch.isfinite(v)].abs().max()) if v.numel() else 0.0
        found.append(r)
    return found


def tolerance(r, d, dtype, kind, tokens):
    """`tokens`: the call has at most 16 query rows to a key head.  out: as serve_util.attention_tolerance (sums, exponentials, what a weight meets the values in).  Tokens over quantised pages: weights
    times scales in fp16, half a step relative, and where that type has no normal number left 2^-25 in units of 2^-7 of the largest such product, times a
    code: keys 2^-31 of the largest value; e2m1 values below 2^-27 of their row's largest scale are nothing (six times that, 2^-24 of the
    largest value at most, with 6 the largest code, and keys whose scores shift as much are inside the logits' error where the data is even)."""
    if dtype == torch.float32 or kind == ROWS:
        return U.attention_tolerance(r, d, dtype)
    if not tokens:                                             # (fp16 or bf16 weights: the coarser; units up to four times the largest values seen)
        return U.attention_tolerance(r, d, dtype) + r["keys"] * 2.0 ** -29 * r["largest"]
    per_weight = 2 * U.logit_error(r["reach"], d) + 2.0 ** -20 + 2 * r["keys"] * 2.0 ** -24 + U.HALF[torch.float16]
    own = per_weight[..., None] * r["weight"] + r["keys"] * 2.0 ** -31 * r["largest"]
    if kind == E2M1:
        own = own + 2.0 ** -24 * r["largest"]
    return own + U.HALF[torch.bfloat16] * (r["out"].abs() + own) + 1e-30


# (kind, heads, key heads, elements, sequences of (queries, rows)) -> (tiles of rows that share what is unpacked, CTAs to a cluster, several clusters to a sequence) of calls on tiles
CLUSTERS = {
    (ROWS, 24, 24, 64, ((20, 600),) * 4): (0, 2, False), (ROWS, 16, 16, 128, ((20, 600),) * 4): (0, 4, False), (ROWS, 2, 2, 96, ((20, 500),)): (0, 8, False),
    (ROWS, 8, 8, 192, ((250, 500),)): (0, 4, False), (ROWS, 8, 8, 256, ((400, 900), (400, 1000), (1, 2))): (0, 2, False), (ROWS, 32, 8, 64, ((400, 9000),)): (0, 4, True),
    (E4M3, 32, 32, 128, ((20, 600),) * 4): (1, 2, False), (E2M1, 16, 16, 64, ((20, 600),) * 4): (1, 4, False), (E4M3, 2, 2, 192, ((20, 500),)): (1, 8, False),
    (E4M3, 16, 16, 128, ((130, 2900), (62, 3000))): (2, 4, False), (E2M1, 32, 32, 64, ((130, 2900), (62, 3000))): (2, 2, False), (E4M3, 4, 1, 128, ((60, 70000),)): (2, 4, True),
    (E4M3, 2, 2, 64, ((130, 500),)): (0, 8, False),
}
