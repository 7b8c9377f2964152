"""A cache in pages, quantised as it is written, as cases that can be timed: writing rows into it, reading them back, and attention over it.

* ``write``   rows of keys and values into pages of the rows' own type (``PruneContext.page_write``);
* ``store``   the same into quantised pages (``page`` = "e4m3": 8 bits, one scale a row and head; "e2m1": 4 bits, one for 32 elements), and
              the rows read back as they are now worth (``page_read``): what a prune point scores when its rows are cached already;
* ``read``    rows of a long or of many caches back as dense rows (``PruneContext.page_read``);
* ``attend``  attention of single tokens or chunks of new tokens over the pages (``PruneContext.page_attention``).

Cached row j of a sequence is row j % page_rows of page table[sequence][j // page_rows]; pages lie in no order. Scales are powers of two, kept
as a byte: 2^(byte - 127). Where ``own`` is false the same is computed by elementary tensor operations in 32 bits.
"""
import random

import numpy as np
import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
_WIDE = {"bf16": 2, "fp32": 4}


def _case(kind, **kw):
    c = {"kind": kind, "dtype": "bf16", "page": "e4m3", "page_rows": 64, "heads": 32, "kv_heads": 8, "head_dim": 128, "batch": 1, "q_lo": 1, "q_hi": 1,
         "past_lo": 0, "past_hi": 0, "window": 0, "sinks": 0, "lse": False, "shape": 0}
    c.update(kw)
    return c


def listed():
    return [
        # One action token of 16 requests into the caches of a deployment without quantisation. All latency.
        _case("write", name="write_token_16", page="rows", batch=16, past_lo=500, past_hi=4000),
        # The prefill of 16 ragged frames, ungrouped keys.
        _case("write", name="write_frames_16", page="rows", kv_heads=32, batch=16, q_lo=768, q_hi=832),
        # The same frames into 8 bits, behind an instruction that is cached already, and their rows as the prune point scores them.
        _case("store", name="store_frames_16_e4m3", batch=16, q_lo=768, q_hi=800, past_lo=17, past_hi=32),
        # A long history into 4 bits and back, small pages.
        _case("store", name="store_long_e2m1", page="e2m1", page_rows=16, q_lo=65537, q_hi=65537),
        # One frame's visual rows back from 8 bits (256 image and 512 point tokens). Latency.
        _case("read", name="read_frame_e4m3", q_lo=768, q_hi=768, past_lo=32, past_hi=32),
        # A long history back from 4 bits.
        _case("read", name="read_long_e2m1", page="e2m1", q_lo=131071, q_hi=131071),
        # One action token of 16 requests over quantised caches of unlike lengths.
        _case("attend", name="attend_token_16_e4m3", batch=16, past_lo=500, past_hi=4000),
        # One token over a long history in 4 bits: bound by the bytes of the cache, or by unpacking them.
        _case("attend", name="attend_token_long_e2m1", page="e2m1", past_lo=131071, past_hi=131071),
        # One token of 16 requests over pruned frames, ungrouped keys, sliding window, pages of the rows' own type.
        _case("attend", name="attend_token_16_rows", page="rows", page_rows=16, kv_heads=32, batch=16, past_lo=1500, past_hi=3000, window=2048, sinks=4),
        # An action chunk (8 steps of 7 values) of 4 requests, decoded at once over 8-bit caches.
        _case("attend", name="attend_chunk_4_e4m3", page_rows=32, batch=4, q_lo=56, q_hi=56, past_lo=2000, past_hi=6000),
        # A chunk of a long prefill: bound by the matrix products.
        _case("attend", name="attend_chunk_long", page="rows", heads=16, kv_heads=4, q_lo=4096, q_hi=4096, past_lo=12289, past_hi=12289, lse=True),
        # The tiny fp32 configuration (16 + 64 + 128 tokens, 8 heads of 64) behind a short cache.
        _case("attend", name="attend_tiny_fp32", dtype="fp32", page="rows", page_rows=16, heads=8, kv_heads=8, head_dim=64, q_lo=208, q_hi=208, past_lo=40,
              past_hi=40, window=64, sinks=2),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm."""
    return int(round(lo * (hi / lo) ** rng.random()))


def _model(rng):
    return rng.choice([{"heads": 32, "kv_heads": 32, "head_dim": 128}, {"heads": 32, "kv_heads": 8, "head_dim": 128},
                       {"heads": 8, "kv_heads": 8, "head_dim": 64}, {"heads": 32, "kv_heads": 32, "head_dim": 96},
                       {"heads": 16, "kv_heads": 16, "head_dim": 256}, {"heads": 16, "kv_heads": 4, "head_dim": 128},
                       {"heads": 12, "kv_heads": 4, "head_dim": 64}, {"heads": 28, "kv_heads": 4, "head_dim": 128},
                       {"heads": 8, "kv_heads": 1, "head_dim": 160}])


def draw(rng):
    kind = rng.choice(["write", "store", "store", "read", "attend", "attend", "attend", "attend"])
    c = {"dtype": rng.choice(["bf16", "bf16", "bf16", "fp32"]), "page_rows": rng.choice([16, 32, 64, 128, 256]), "shape": rng.randrange(1, 1 << 20),
         **_model(rng)}
    c["page"] = "rows" if kind == "write" else rng.choice(["e4m3", "e2m1"]) if kind == "store" else rng.choice(["rows", "e4m3", "e2m1"])
    if kind != "attend":
        batch = _log(rng, 1, 32)
        hi = _log(rng, 1, 8192 // batch)
        past = rng.choice([0, _log(rng, 1, 512)])
        return _case(kind, batch=batch, q_lo=max(1, hi // 2), q_hi=hi, past_lo=past // 2, past_hi=past, **c)
    c.update(window=rng.choice([0, 0, _log(rng, 16, 4096)]), sinks=rng.choice([0, 1, 4, 16]), lse=rng.random() < 0.3)
    form = rng.choice(["prefill", "token", "token", "chunk"])
    if form == "prefill":
        batch = _log(rng, 1, 8)
        hi = _log(rng, 2, 2000 // batch)
        past = rng.choice([0, _log(rng, 1, 2000 // batch)])
        return _case(kind, batch=batch, q_lo=max(1, int(hi * rng.uniform(0.4, 1.0))), q_hi=hi, past_lo=past // 2, past_hi=past, **c)
    batch = _log(rng, 1, 32)
    past = _log(rng, 16, max(64, 65536 // batch) if form == "token" else 4096)
    n = 1 if form == "token" else _log(rng, 2, 200)
    return _case(kind, batch=batch if form == "token" else min(batch, 4), q_lo=max(1, n // 2), q_hi=n, past_lo=max(1, past // 2), past_hi=past, **c)


# ---- what the shapes of a case are (the same for every seed)


def _shape(case):
    """New rows, cached rows (those among them), and first new row of every sequence."""
    rng = np.random.default_rng(case["shape"])
    nq = rng.integers(case["q_lo"], case["q_hi"] + 1, case["batch"])
    nkv = rng.integers(case["past_lo"], case["past_hi"] + 1, case["batch"]) + nq
    return nq, nkv, np.concatenate([[0], np.cumsum(nq)[:-1]])


def _row_bytes(case):
    """Bytes of a cached row of one head, its scales among them."""
    d = case["head_dim"]
    return {"rows": d * _WIDE[case["dtype"]], "e4m3": d + 1, "e2m1": d // 2 + d // 32}[case["page"]]


def _visible(case):
    """(visible (query, row) pairs, rows that some query sees) of one head."""
    nq, nkv, _ = _shape(case)
    window = case["window"] or 1 << 30
    pairs = rows = 0
    for a, b in zip(nq, nkv):
        p = np.arange(b - a, b, dtype=np.int64)
        low = np.maximum(p - window + 1, 0)
        pairs += int((p + 1 - low + np.minimum(case["sinks"], low)).sum())
        rows += int(b - low.min() + min(case["sinks"], low.min()))
    return pairs, rows, int(nq.sum())


def work(case):
    H, G, d = case["heads"], case["kv_heads"], case["head_dim"]
    wide = d * _WIDE[case["dtype"]]
    if case["kind"] == "attend":
        pairs, rows, queries = _visible(case)
        return {"bytes": 2 * queries * H * wide + 2 * rows * G * _row_bytes(case), "flops": 4 * d * H * pairs}
    values = 2 * G * int(_shape(case)[0].sum())               # rows of one head, keys and values
    moved = wide + _row_bytes(case)
    if case["kind"] == "store":                               # into the pages; out of them; the dense rows
        moved = 2 * wide + 2 * _row_bytes(case)
    return {"bytes": values * moved, "flops": values * d * (2 if case["kind"] == "store" else 1)}


# ---- inputs


def _normal(gen, *shape, dtype="bf16"):
    return torch.randn(*shape, generator=gen, device="cuda").to(_TYPES[dtype])


def _channels(gen, *shape):
    """Keys have channels that are larger than the others, as rotated keys do."""
    return torch.exp(torch.randn(*shape, generator=gen, device="cuda") * 0.7)


def _pow2(e):
    """2^e for whole numbers e in [-126, 127]."""
    return ((e + 127) << 23).view(torch.float32)


def _quantise(x, page):
    """Codes (as they are stored) and scale bytes of rows [..., d], 32 bits."""
    g = x.shape[-1] if page == "e4m3" else 32
    x = x.unflatten(-1, (-1, g))
    big = x.abs().amax(-1)
    m, e = torch.frexp(big)
    e = e - 9 + (m > 0.875) if page == "e4m3" else e - 3 + (m > 0.75)          # 448 = 0.875 * 2^9, 6 = 0.75 * 2^3
    e = torch.where(big > 0, e, -117).clamp(-117, 119 if page == "e4m3" else 125).to(torch.int32)
    y = (x * _pow2(-e)[..., None]).flatten(-2)
    scale = (e + 127).to(torch.uint8)
    if page == "e4m3":
        return y.clamp(-448, 448).to(torch.float8_e4m3fn), scale.squeeze(-1)
    a = y.abs()
    code = torch.zeros_like(a, dtype=torch.uint8)
    for at, tie in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (a >= at) if tie else (a > at)
    code |= torch.signbit(y).to(torch.uint8) << 3
    return code[..., 0::2] | code[..., 1::2] << 4, scale


def _values(codes, scale, page):
    """What codes and scale bytes stand for, 32 bits."""
    if page == "rows":
        return codes.float()
    if page == "e4m3":
        return codes.float() * _pow2(scale.int() - 127)[..., None]
    steps = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=codes.device)
    steps = torch.cat([steps, -steps])
    y = torch.stack([steps[(codes & 15).int()], steps[(codes >> 4).int()]], -1).flatten(-2)
    return (y.unflatten(-1, (-1, 32)) * _pow2(scale.int() - 127)[..., None]).flatten(-2)


def _bits(x):
    return x.view(torch.uint8)


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    H, G, d, P = case["heads"], case["kv_heads"], case["head_dim"], case["page_rows"]
    nq, nkv, q_row = _shape(case)
    batch = case["batch"]
    need = -(-nkv // P)
    n_pages = int(need.sum()) + 3                             # (a pool holds other pages too)
    order = torch.randperm(n_pages, generator=gen, device="cuda", dtype=torch.int64).to(torch.int32)
    table = torch.full((batch, int(need.max())), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b in range(batch):
        table[b, :need[b]] = order[at:at + need[b]]
        at += int(need[b])
    s = {"case": case, "table": table, "lengths": (nq, nkv, q_row)}
    rows = int(nq.sum())
    if case["kind"] in ("write", "store"):
        fused = _normal(gen, rows, (H + 2 * G) * d, dtype=case["dtype"])                # the projection that values are a part of
        s["new_k"] = (_normal(gen, rows, G, d, dtype="fp32") * _channels(gen, G, d)).to(_TYPES[case["dtype"]])
        s["new_v"] = fused[:, (H + G) * d:].unflatten(1, (G, d))
        width = d // 2 if case["page"] == "e2m1" else d
        kept = {"rows": _TYPES[case["dtype"]], "e4m3": torch.float8_e4m3fn, "e2m1": torch.uint8}[case["page"]]
        for n in ("k", "v"):
            s[n] = torch.zeros(n_pages, G, P, width, device="cuda").to(kept)
            scales = {"rows": None, "e4m3": (n_pages, G, P), "e2m1": (n_pages, G, P, d // 32)}[case["page"]]
            s[n + "_scale"] = None if scales is None else torch.zeros(scales, dtype=torch.uint8, device="cuda")
    else:
        for n in ("k", "v"):
            x = torch.randn(n_pages, G, P, d, generator=gen, device="cuda")
            if n == "k":
                x *= _channels(gen, G, 1, d)
                x *= 1 + (torch.rand(n_pages, 1, P, 1, generator=gen, device="cuda") < 0.05)        # a few keys that draw attention
            x = x.to(_TYPES[case["dtype"]])
            s[n], s[n + "_scale"] = (x, None) if case["page"] == "rows" else _quantise(x.float(), case["page"])
        if case["kind"] == "attend":
            s["q"] = _normal(gen, rows, H, d, dtype=case["dtype"])
            s["lse"] = torch.zeros(rows, H, device="cuda") if case["lse"] else None
    if own:
        from paper_2604_09244_b200 import mvla
        s["ctx"] = mvla.PruneContext(dtype=_TYPES[case["dtype"]], n_heads=H, head_dim=d, d_model=H * d, max_batch=batch, max_text=32,
                                     max_2d=256, max_3d=512, n_kv_heads=G)
        s["pool"] = mvla.PagePool(k=s["k"], v=s["v"], k_scale=s["k_scale"], v_scale=s["v_scale"])
        s["seqs"] = mvla.c_seqs([mvla.Seq(q_row=int(r), n_q=int(a), n_kv=int(b)) for r, a, b in zip(q_row, nq, nkv)])
    return s


# ---- one pass


def run(s):
    kind = s["case"]["kind"]
    if not own:
        return {"write": _plain_write, "store": _plain_store, "read": _plain_read, "attend": _plain_attend}[kind](s)
    c, ctx, pool, seqs, table = s["case"], s["ctx"], s["pool"], s["seqs"], s["table"]
    if kind == "attend":
        out = ctx.page_attention(pool, seqs, table, s["q"], window=c["window"] or None, n_sink=c["sinks"], lse=s["lse"])
        return {"out": out, "lse": s["lse"]}
    if kind != "read":
        ctx.page_write(pool, seqs, table, s["new_k"], s["new_v"])
    if kind == "write":
        return {"k": s["k"], "v": s["v"]}
    k, v = ctx.page_read(pool, seqs, table)
    return {"k": k, "v": v}


def _places(s):
    """Page and row inside it of every new row, packed over the sequences."""
    nq, nkv, _ = (torch.from_numpy(x).cuda() for x in s["lengths"])
    b = torch.repeat_interleave(torch.arange(len(nq), device="cuda"), nq)
    i = torch.arange(len(b), device="cuda") - (nq.cumsum(0) - nq)[b]
    j = (nkv - nq)[b] + i
    P = s["case"]["page_rows"]
    return s["table"].long()[b, j // P], j % P


def _plain_write(s):
    page, row = _places(s)
    for n in ("k", "v"):
        if s["case"]["page"] == "rows":
            s[n][page, :, row] = s["new_" + n]
        else:
            codes, scale = _quantise(s["new_" + n].float(), s["case"]["page"])
            _bits(s[n])[page, :, row] = _bits(codes)
            s[n + "_scale"][page, :, row] = scale
    return {"k": s["k"], "v": s["v"]}


def _plain_read(s):
    page, row = _places(s)
    kind, wide = s["case"]["page"], _TYPES[s["case"]["dtype"]]
    out = {}
    for n in ("k", "v"):
        codes = _bits(s[n])[page, :, row].view(s[n].dtype)
        scale = None if kind == "rows" else s[n + "_scale"][page, :, row]
        out[n] = _values(codes, scale, kind).to(wide)
    return out


def _plain_store(s):
    _plain_write(s)
    return _plain_read(s)


def _plain_attend(s):
    c = s["case"]
    H, G, d, P = c["heads"], c["kv_heads"], c["head_dim"], c["page_rows"]
    nq, nkv, q_row = (torch.from_numpy(x).cuda() for x in s["lengths"])
    i, j = torch.arange(int(nq.max()), device="cuda")[None], torch.arange(int(nkv.max()), device="cuda")[None]
    q_there, k_there = i < nq[:, None], j < nkv[:, None]
    qi = torch.where(q_there, q_row[:, None] + i, 0)
    page = s["table"].long().gather(1, (j // P).expand(len(nq), -1)).clamp_min(0)
    row = (j % P).expand(len(nq), -1)

    def dense(n):                                             # [batch, rows, G, d], 32 bits
        codes = _bits(s[n])[page, :, row].view(s[n].dtype)
        return _values(codes, None if c["page"] == "rows" else s[n + "_scale"][page, :, row], c["page"])

    p = (nkv - nq)[:, None] + i
    back = p[:, :, None] - j[:, None, :]
    seen = (back >= 0) & q_there[:, :, None] & k_there[:, None, :]
    if c["window"]:
        seen &= (back < c["window"]) | (j < c["sinks"])[:, None, :]
    q = s["q"].float()[qi].unflatten(2, (G, H // G)).permute(0, 2, 3, 1, 4).flatten(2, 3)       # [batch, G, H/G q, d]
    logits = (q @ dense("k").permute(0, 2, 3, 1)).mul_(d ** -0.5).unflatten(2, (H // G, -1))
    logits.masked_fill_(~seen[:, None, None], float("-inf"))
    top = logits.amax(-1, keepdim=True)
    top = torch.where(top == float("-inf"), 0.0, top)
    w = logits.sub_(top).exp_()
    total = w.sum(-1, keepdim=True)
    w.div_(torch.where(total > 0, total, 1.0))
    v = torch.where(k_there[:, :, None, None], dense("v"), 0.0).permute(0, 2, 1, 3)
    o = (w.flatten(2, 3) @ v).unflatten(2, (H // G, -1)).permute(0, 3, 1, 2, 4).flatten(2, 3)   # [batch, q, H, d]
    out = torch.zeros(s["q"].shape, dtype=_TYPES[c["dtype"]], device="cuda")
    out[qi[q_there]] = o[q_there].to(out.dtype)
    if s["lse"] is not None:
        s["lse"][qi[q_there]] = (total.log() + top).squeeze(-1).permute(0, 3, 1, 2).flatten(2, 3)[q_there]
    return {"out": out, "lse": s["lse"]}


# ---- the definitions in 64 bits


def exact(case, seed):
    global own
    before, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = before
    return {"write": _exact_write, "store": _exact_store, "read": _exact_read, "attend": _exact_attend}[case["kind"]](s)


def _exact_rows(s, name, b):
    """The cached rows of sequence b [rows, G, d]: bit fields of the codes, times their scale."""
    kind, P = s["case"]["page"], s["case"]["page_rows"]
    n = int(s["lengths"][1][b])
    pages = s["table"][b, : -(-n // P)].long()
    flat = lambda x: x[pages].transpose(1, 2).flatten(0, 1)[:n]  # noqa: E731   [rows, G, ...]
    if kind == "rows":
        return flat(s[name]).double()
    scale = torch.exp2(flat(s[name + "_scale"]).double() - 127)
    code = flat(_bits(s[name])).long()
    if kind == "e4m3":
        e, m = code >> 3 & 15, (code & 7).double()
        x = torch.where(e > 0, (1 + m / 8) * torch.exp2(e.double() - 7), m / 8 * 2.0 ** -6)
        return torch.where(code > 127, -x, x) * scale[..., None]
    code = torch.stack([code % 16, code // 16], -1).flatten(-2)
    e, m = code >> 1 & 3, (code & 1).double()
    x = torch.where(e > 0, (1 + m / 2) * torch.exp2(e.double() - 1), m / 2)
    return torch.where(code > 7, -x, x) * scale.repeat_interleave(32, -1)


def _exact_write(s):
    P = s["case"]["page_rows"]
    out = {}
    for n in ("k", "v"):
        pool = s[n].double()
        for a, b, r, pages in zip(*(x.tolist() for x in s["lengths"]), s["table"].tolist()):
            i = 0
            while i < a:                                      # runs of rows inside a page
                j = b - a + i
                m = min(P - j % P, a - i)
                pool[pages[j // P], :, j % P:j % P + m] = s["new_" + n][r + i:r + i + m].double().transpose(0, 1)
                i += m
        out[n] = pool
    return out


def _exact_store(s):
    e4m3 = s["case"]["page"] == "e4m3"
    top, bits, least = (448.0, 3, -6) if e4m3 else (6.0, 1, 0)
    out = {}
    for n in ("k", "v"):
        x = s["new_" + n].double()
        x = x.unflatten(-1, (-1, x.shape[-1] if e4m3 else 32))
        big = x.abs().amax(-1, keepdim=True)
        scale = torch.exp2(torch.ceil(torch.log2(big.clamp_min(1e-300) / top)).clamp(-117, 119 if e4m3 else 125))
        scale = torch.where(scale * top < big, scale * 2, torch.where(scale * top / 2 >= big, scale / 2, scale)).clamp_min(2.0 ** -117)
        y = x / scale
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** least))) - bits)
        out[n] = ((y / step).round() * step).clamp(-top, top).mul(scale).flatten(-2)
    return out


def _exact_read(s):
    nq, nkv, _ = s["lengths"]
    return {n: torch.cat([_exact_rows(s, n, b)[nkv[b] - nq[b]:] for b in range(len(nq))]) for n in ("k", "v")}


def _exact_attend(s):
    c = s["case"]
    H, G, d = c["heads"], c["kv_heads"], c["head_dim"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(out.shape[:2], dtype=torch.float64, device="cuda")
    for b, (a, n, r) in enumerate(zip(*(x.tolist() for x in s["lengths"]))):
        k, v = _exact_rows(s, "k", b), _exact_rows(s, "v", b)
        p, j = torch.arange(n - a, n, device="cuda"), torch.arange(n, device="cuda")
        blocked = j[None, :] > p[:, None]
        if c["window"]:
            blocked |= (j[None, :] <= p[:, None] - c["window"]) & (j[None, :] >= c["sinks"])
        for h in range(H):
            g = h * G // H
            l = s["q"][r:r + a, h].double() @ k[:, g].T / d ** 0.5
            l[blocked] = float("-inf")
            z = torch.logsumexp(l, 1)
            lse[r:r + a, h] = z
            out[r:r + a, h] = torch.exp(l - z[:, None]) @ v[:, g]
    return {"out": out, "lse": lse if s["lse"] is not None else None}
