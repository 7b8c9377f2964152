"""The operators around a prune point, as cases that can be timed: what makes the query and key rows that pruning scores, the
attention over the rows that survive, and the eviction that keeps a cache small while action tokens are decoded.

* ``rope``    norms of queries and keys for each head and the position rotation (``PruneContext.qk_norm_rope``): the projections'
              rows, as slices of one fused tensor, become query rows and rows of the key / value cache;
* ``attend``  attention with a sliding window and sinks (``PruneContext.window_attention``) over packed rows or a cache, positions
              counted (``pos`` = "count"), those of rows that a prune step kept ("kept": ascending, with gaps) or those of a cache
              whose holes were filled ("filled": in no order); with ``mass`` the weights are added up for every cached row;
* ``evict``   eviction by that accumulated weight (``PruneContext.cache_evict``): keys and values move in place, positions and
              weights into arrays of their own.

Where ``own`` is false the same is computed by elementary tensor operations in 32 bits.
"""
import random

import numpy as np
import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32, "fp8": torch.float8_e4m3fn}
_BYTES = {"bf16": 2, "fp32": 4, "fp8": 1}


def _rope(**kw):
    c = {"kind": "rope", "dtype": "bf16", "heads": 32, "kv_heads": 32, "head_dim": 128, "rows": 16, "rot_dim": 128,
         "interleaved": False, "far": 4096, "spare": 0, "shape": 0}
    c.update(kw)
    return c


def _attend(**kw):
    c = {"kind": "attend", "dtype": "bf16", "heads": 32, "kv_heads": 32, "head_dim": 128, "batch": 1, "q_lo": 1, "q_hi": 1,
         "past_lo": 0, "past_hi": 0, "window": 0, "sinks": 0, "pos": "count", "mass": False, "lse": False, "shape": 0}
    c.update(kw)
    return c


def _evict(**kw):
    c = {"kind": "evict", "dtype": "bf16", "heads": 32, "kv_heads": 8, "head_dim": 128, "batch": 1, "len_lo": 1025, "len_hi": 1025,
         "keep_lo": 1.0, "keep_hi": 1.0, "over": 0, "sinks": 4, "recent": 128, "shape": 0}
    c.update(kw)
    return c


def listed():
    return [
        # One decoded action token of 16 requests: their rows into the cache.  All latency.
        _rope(name="rope_token_16", rows=16, spare=240),
        # The prefill of 16 frames with 32 text, 256 image and 512 point tokens.
        _rope(name="rope_prefill_16", rows=12800),
        # A quantised deployment with grouped keys: bf16 projections become e4m3 rows; far positions, pairs side by side, half the head.
        _rope(name="rope_fp8_grouped", dtype="fp8", kv_heads=8, rows=4099, rot_dim=64, interleaved=True, far=1000000),
        # The rows that one pruned frame keeps (32 text + 102 + 154), after the prune point: the smallest prefill.
        _attend(name="attend_pruned_frame", q_lo=288, q_hi=288, pos="kept", window=512, sinks=4),
        # The prefill of a ragged batch of 16 frames with accumulated weights, which eviction needs later.
        _attend(name="attend_prefill_16", batch=16, q_lo=784, q_hi=832, window=512, sinks=4, mass=True),
        # A long instruction history, grouped heads, everything before a token visible: bound by the matrix products.
        _attend(name="attend_long", heads=16, kv_heads=4, q_lo=8192, q_hi=8192, lse=True),
        # The tiny fp32 configuration (16 + 64 + 128 tokens, 8 heads of 64).
        _attend(name="attend_tiny_fp32", dtype="fp32", heads=8, kv_heads=8, head_dim=64, q_lo=208, q_hi=208, window=64, sinks=2),
        # One action token of 16 requests over caches that eviction has run on, grouped e4m3 keys, weights added up.
        _attend(name="attend_token_16_fp8", dtype="fp8", kv_heads=8, batch=16, past_lo=500, past_hi=4000, pos="filled", window=2048,
                sinks=4, mass=True),
        # One token over a long history: bound by the bytes of the cache.
        _attend(name="attend_token_long", kv_heads=8, past_lo=131071, past_hi=131071),
        # A decode step's eviction: 16 caches that are one row over their budget.
        _evict(name="evict_step_16", batch=16, over=1),
        # The eviction after a prefill of 16 frames, ungrouped keys: three rows of ten stay.
        _evict(name="evict_frames_16", kv_heads=32, batch=16, len_lo=784, len_hi=832, keep_lo=0.25, keep_hi=0.35, recent=32),
        # A long history cut to an eighth.
        _evict(name="evict_long", len_lo=65537, len_hi=65537, keep_lo=0.125, keep_hi=0.125),
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
    kind = rng.choice(["rope", "attend", "attend", "attend", "evict"])
    m = _model(rng)
    dtype = rng.choice(["bf16", "bf16", "fp8", "fp32"])
    shape = rng.randrange(1, 1 << 20)
    if kind == "rope":
        return _rope(dtype=dtype, rows=_log(rng, 1, 6000), rot_dim=rng.choice([32, m["head_dim"] // 32 * 16, m["head_dim"]]),
                     interleaved=rng.random() < 0.3, far=_log(rng, 512, 2000000), spare=rng.choice([0, 0, 64]), shape=shape, **m)
    if kind == "evict":
        batch = _log(rng, 1, 16)
        hi = _log(rng, 64, max(128, 24576 // batch))
        keep = rng.uniform(0.1, 0.9)
        return _evict(dtype=dtype, batch=batch, len_lo=max(40, hi // 2), len_hi=hi, keep_lo=keep * 0.9, keep_hi=keep,
                      over=rng.choice([0, 0, 1]), sinks=rng.choice([0, 1, 4, 8]), recent=_log(rng, 1, max(2, hi // 32)), shape=shape, **m)
    c = {"dtype": dtype, "window": rng.choice([0, _log(rng, 16, 4096)]), "sinks": rng.choice([0, 1, 4, 16]),
         "mass": rng.random() < 0.4, "lse": rng.random() < 0.3, "shape": shape, **m}
    form = rng.choice(["prefill", "token", "token", "chunk"])
    if form == "prefill":
        batch = _log(rng, 1, 16)
        hi = _log(rng, 2, 3000 if batch == 1 else 1000)
        return _attend(batch=batch, q_lo=max(1, int(hi * rng.uniform(0.4, 1.0))), q_hi=hi, pos=rng.choice(["count", "kept"]), **c)
    batch = _log(rng, 1, 32)
    past = _log(rng, 16, max(64, 65536 // batch) if form == "token" else 4096)
    n = 1 if form == "token" else _log(rng, 2, 200)
    return _attend(batch=batch if form == "token" else min(batch, 4), q_lo=max(1, n // 2), q_hi=n, past_lo=max(1, past // 2),
                   past_hi=past, pos=rng.choice(["count", "kept", "filled"]), **c)


# ---- what the shapes of a case are (lengths and positions: the same for every seed)


def _positions(rng, n):
    """Positions of n rows that a prune step kept: ascending, with gaps."""
    return np.sort(rng.choice(int(n * 1.5) + 8, size=n, replace=False)).astype(np.int32)


def _attend_shape(case):
    rng = np.random.default_rng(case["shape"])
    nq = rng.integers(case["q_lo"], case["q_hi"] + 1, case["batch"])
    nkv = rng.integers(case["past_lo"], case["past_hi"] + 1, case["batch"]) + nq
    gap = rng.integers(0, 3, case["batch"])                    # rows between the sequences that belong to none
    q_row = np.concatenate([[0], np.cumsum(nq)[:-1]])
    kv_row = np.concatenate([[0], np.cumsum(nkv + gap)[:-1]])
    q_pos, kv_pos = [], []
    for a, b, g in zip(nq, nkv, gap):
        p = np.arange(b, dtype=np.int32) if case["pos"] == "count" else _positions(rng, b)
        q_pos.append(p[b - a:])
        if case["pos"] == "filled" and b > a:
            p = np.concatenate([p[:b - a][_order(rng, b - a)], p[b - a:]])
        kv_pos += [p, np.full(g, -1, np.int32)]
    return nq, nkv, q_row, kv_row, np.concatenate(q_pos), np.concatenate(kv_pos)


def _order(rng, n):
    """The order of rows in a cache whose holes were filled: most rows in place, every third somewhere else."""
    o = np.arange(n)
    some = rng.permutation(n)[: n // 3]
    o[np.sort(some)] = some
    return o


def _evict_shape(case):
    rng = np.random.default_rng(case["shape"])
    n = rng.integers(case["len_lo"], case["len_hi"] + 1, case["batch"])
    keep = rng.uniform(case["keep_lo"], case["keep_hi"], case["batch"])
    least = case["sinks"] + case["recent"]
    budget = np.maximum(least, n - 1 if case["over"] else np.floor(n * keep).astype(np.int64))
    row = np.concatenate([[0], np.cumsum(n)[:-1]])
    pos = np.concatenate([np.arange(m, dtype=np.int32)[_order(rng, m)] if case["over"] else np.arange(m, dtype=np.int32) for m in n])
    return n, budget, row, pos


def _visible(case):
    """(visible (query, key) pairs, key rows that some query sees) of an ``attend`` case, one head."""
    nq, nkv, q_row, kv_row, q_pos, kv_pos = _attend_shape(case)
    window = case["window"] or 1 << 30
    pairs = rows = 0
    for a, b, r, s in zip(nq, nkv, q_row, kv_row):
        p, kp = q_pos[r:r + a].astype(np.int64), np.sort(kv_pos[s:s + b]).astype(np.int64)
        upto = np.searchsorted(kp, p, "right")
        low = np.searchsorted(kp, p - window, "right")
        sink = np.minimum(np.searchsorted(kp, min(case["sinks"], 1 << 30), "left"), upto)
        pairs += int((upto - low + np.minimum(sink, low)).sum())
        first = int(low.min())
        rows += int(upto.max()) - first + min(first, int(sink.max()))
    return pairs, rows, int(nq.sum())


def work(case):
    e, H, G, d = _BYTES[case["dtype"]], case["heads"], case["kv_heads"], case["head_dim"]
    if case["kind"] == "rope":
        wide = 4 if case["dtype"] == "fp32" else 2
        values = case["rows"] * (H + 2 * G) * d
        return {"bytes": values * (wide + e) + 4 * case["rows"], "flops": case["rows"] * (H + G) * (4 * d + 4 * case["rot_dim"])}
    if case["kind"] == "evict":
        n, budget, row, pos = _evict_shape(case)
        new = np.minimum(n, budget)
        moved = (1 - new / n) * new                            # survivors lie anywhere with equal chances
        return {"bytes": int(8 * n.sum() + 12 * new.sum() + 4 * G * d * e * moved.sum()), "flops": int(n.sum())}
    pairs, rows, queries = _visible(case)
    wide = 4 if case["dtype"] == "fp32" else 2
    read = queries * H * d * (e + wide) + 2 * rows * G * d * e
    return {"bytes": read + (8 * rows if case["mass"] else 0), "flops": 4 * d * H * pairs}


# ---- inputs


def _normal(gen, *shape, dtype="bf16"):
    x = torch.randn(*shape, generator=gen, device="cuda")
    return x.clamp(-440, 440).to(_TYPES[dtype])


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    H, G, d = case["heads"], case["kv_heads"], case["head_dim"]
    s = {"case": case}
    if case["kind"] == "rope":
        rows = case["rows"]
        wide = "fp32" if case["dtype"] == "fp32" else "bf16"
        s["qkv"] = _normal(gen, rows, (H + 2 * G) * d, dtype=wide)          # the fused projection
        s["q_weight"] = (1 + 0.1 * torch.randn(d, generator=gen, device="cuda")).to(_TYPES[wide])
        s["k_weight"] = (1 + 0.1 * torch.randn(d, generator=gen, device="cuda")).to(_TYPES[wide])
        s["pos"] = torch.randint(0, case["far"], (rows,), generator=gen, device="cuda", dtype=torch.int32)
        s["inv_freq"] = 10000.0 ** (-torch.arange(0, case["rot_dim"], 2, device="cuda", dtype=torch.float64) / case["rot_dim"])
        cached = rows + case["spare"]                                        # rows of the cache, in the order that its allocator gave
        s["out_rows"] = torch.randperm(cached, generator=gen, device="cuda", dtype=torch.int64)[:rows].to(torch.int32)
        s["k_cache"] = torch.zeros(cached, G, d, device="cuda").to(_TYPES[case["dtype"]])
        s["v_cache"] = torch.zeros(cached, G, d, device="cuda").to(_TYPES[case["dtype"]])
        batch = 1
    elif case["kind"] == "attend":
        nq, nkv, q_row, kv_row, q_pos, kv_pos = _attend_shape(case)
        s["q"] = _normal(gen, int(nq.sum()), H, d, dtype=case["dtype"])
        rows = len(kv_pos)
        s["k"], s["v"] = _normal(gen, rows, G, d, dtype=case["dtype"]), _normal(gen, rows, G, d, dtype=case["dtype"])
        hot = torch.rand(rows, 1, 1, generator=gen, device="cuda") < 0.05    # a few keys that draw attention, as salient tokens do
        s["k"] = torch.where(hot, s["k"].float() * 2, s["k"].float()).clamp(-440, 440).to(_TYPES[case["dtype"]])
        s["q_pos"], s["kv_pos"] = (None, None) if case["pos"] == "count" else (dev(q_pos), dev(kv_pos))
        s["mass"] = torch.rand(rows, generator=gen, device="cuda") if case["mass"] else None
        s["lse"] = torch.zeros(int(nq.sum()), H, device="cuda") if case["lse"] else None
        s["lengths"] = nq, nkv, q_row, kv_row
        batch = case["batch"]
    else:
        n, budget, row, pos = _evict_shape(case)
        rows = int(n.sum())
        s["k"], s["v"] = _normal(gen, rows, G, d, dtype=case["dtype"]), _normal(gen, rows, G, d, dtype=case["dtype"])
        s["mass"] = torch.rand(rows, generator=gen, device="cuda").clamp_min(1e-6).log().neg().square()
        s["pos"] = dev(pos)
        s["pos_out"] = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
        s["mass_out"] = torch.zeros(rows, device="cuda")
        s["kept"] = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
        s["lengths"] = n, budget, row
        batch = case["batch"]
    if own:
        from paper_2604_09244_b200 import mvla
        s["ctx"] = mvla.PruneContext(dtype=_TYPES[case["dtype"]], n_heads=H, head_dim=d, d_model=H * d, max_batch=batch, max_text=32,
                                     max_2d=256, max_3d=512, n_kv_heads=G)
        if case["kind"] == "attend":
            s["seqs"] = mvla.c_seqs([mvla.Seq(q_row=int(a), n_q=int(b), kv_row=int(c), n_kv=int(e))
                                     for a, b, c, e in zip(q_row, nq, kv_row, nkv)])
        elif case["kind"] == "evict":
            s["seqs"] = mvla.c_seqs([mvla.Seq(kv_row=int(a), n_kv=int(b), budget=int(c)) for a, b, c in zip(row, n, budget)])
    return s


# ---- one pass


def _split(s):
    c = s["case"]
    H, G, d = c["heads"], c["kv_heads"], c["head_dim"]
    n = s["qkv"].shape[0]
    q, k, v = s["qkv"].split([H * d, G * d, G * d], dim=1)
    return q.unflatten(1, (H, d)), k.unflatten(1, (G, d)), v.unflatten(1, (G, d)), n


def run(s):
    c = s["case"]
    if not own:
        return {"rope": _plain_rope, "attend": _plain_attend, "evict": _plain_evict}[c["kind"]](s)
    ctx = s["ctx"]
    if c["kind"] == "rope":
        q, k, v, _ = _split(s)
        q_out, k_out, v_out = ctx.qk_norm_rope(q, k, s["pos"], s["inv_freq"], v=v, q_weight=s["q_weight"], k_weight=s["k_weight"],
                                               eps=1e-6, interleaved=c["interleaved"], k_out=s["k_cache"], v_out=s["v_cache"],
                                               out_rows=s["out_rows"])
        return {"q": q_out, "k": k_out, "v": v_out}
    if c["kind"] == "attend":
        out = ctx.window_attention(s["seqs"], s["q"], s["k"], s["v"], window=c["window"] or None, n_sink=c["sinks"], q_pos=s["q_pos"],
                                   kv_pos=s["kv_pos"], lse=s["lse"], mass=s["mass"])
        return {"out": out, "lse": s["lse"], "mass": s["mass"]}
    ctx.cache_evict(s["seqs"], s["k"], s["v"], s["pos"], s["mass"], n_sink=c["sinks"], n_recent=c["recent"], pos_out=s["pos_out"],
                    mass_out=s["mass_out"], kept_idx=s["kept"])
    return {"k": s["k"], "v": s["v"], "pos": s["pos_out"], "mass": s["mass_out"], "kept": s["kept"]}


def _narrow(x, dtype):
    """Rounded once to the type that is kept (e4m3 saturates)."""
    return x.clamp(-448, 448).to(dtype) if dtype == torch.float8_e4m3fn else x.to(dtype)


def _bits(x):
    return x.view(torch.uint8)


def _plain_rope(s):
    c = s["case"]
    q, k, v, n = _split(s)
    r, kind = c["rot_dim"], _TYPES[c["dtype"]]
    angle = s["pos"].double()[:, None] * s["inv_freq"][None, :]
    cos, sin = angle.cos().float()[:, None, :], angle.sin().float()[:, None, :]

    def turn(x, w):
        x = x.float()
        y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.float()
        a, b = (y[..., 0:r:2], y[..., 1:r:2]) if c["interleaved"] else (y[..., :r // 2], y[..., r // 2:r])
        a, b = a * cos - b * sin, b * cos + a * sin
        turned = torch.stack([a, b], -1).flatten(-2) if c["interleaved"] else torch.cat([a, b], -1)
        return _narrow(torch.cat([turned, y[..., r:]], -1), kind)

    at = s["out_rows"].long()
    _bits(s["k_cache"])[at] = _bits(turn(k, s["k_weight"]))
    _bits(s["v_cache"])[at] = _bits(_narrow(v, kind).contiguous())
    return {"q": turn(q, s["q_weight"]), "k": s["k_cache"], "v": s["v_cache"]}


def _padded(row, n):
    """Row numbers [batch, longest] of the sequences, and which of them exist."""
    row, n = torch.from_numpy(np.asarray(row)).cuda(), torch.from_numpy(np.asarray(n)).cuda()
    i = torch.arange(int(n.max()), device="cuda")[None, :]
    there = i < n[:, None]
    return torch.where(there, row[:, None] + i, 0), there


def _plain_attend(s):
    c = s["case"]
    H, G, d = c["heads"], c["kv_heads"], c["head_dim"]
    nq, nkv, q_row, kv_row = s["lengths"]
    qi, q_there = _padded(q_row, nq)
    ki, k_there = _padded(kv_row, nkv)
    if s["q_pos"] is None:
        kp = torch.where(k_there, torch.arange(ki.shape[1], device="cuda")[None, :], -1)
        qp = torch.from_numpy(nkv - nq).cuda()[:, None] + torch.arange(qi.shape[1], device="cuda")[None, :]
    else:
        kp, qp = torch.where(k_there, s["kv_pos"][ki].long(), -1), s["q_pos"][qi].long()
    back = qp[:, :, None] - kp[:, None, :]
    seen = (back >= 0) & (kp >= 0)[:, None, :] & q_there[:, :, None]
    if c["window"]:
        seen &= (back < c["window"]) | (kp < c["sinks"])[:, None, :]
    q = s["q"].float()[qi].unflatten(2, (G, H // G)).permute(0, 2, 3, 1, 4).flatten(2, 3)       # [batch, G, H/G q, d]
    k = s["k"].float()[ki].permute(0, 2, 3, 1)                                                  # [batch, G, d, k]
    v = torch.where(k_there[:, :, None, None], s["v"].float()[ki], 0.0).permute(0, 2, 1, 3)     # [batch, G, k, d]
    logits = (q @ k).mul_(d ** -0.5).unflatten(2, (H // G, -1))
    logits.masked_fill_(~seen[:, None, None], float("-inf"))
    top = logits.amax(-1, keepdim=True)
    top = torch.where(top == float("-inf"), 0.0, top)
    p = logits.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    p.div_(torch.where(total > 0, total, 1.0))
    o = (p.flatten(2, 3) @ v).unflatten(2, (H // G, -1)).permute(0, 3, 1, 2, 4).flatten(2, 3)   # [batch, q, H, d]
    wide = torch.float32 if c["dtype"] == "fp32" else torch.bfloat16
    out = torch.zeros(s["q"].shape, dtype=wide, device="cuda")
    out[qi[q_there]] = o[q_there].to(wide)
    if s["lse"] is not None:
        lse = (total.log() + top).squeeze(-1).permute(0, 3, 1, 2).flatten(2, 3)
        s["lse"][qi[q_there]] = lse[q_there]
    if s["mass"] is not None:
        s["mass"][ki[k_there]] += (p.sum((1, 2, 3)) / H)[k_there]
    return {"out": out, "lse": s["lse"], "mass": s["mass"]}


def _plain_evict(s):
    c = s["case"]
    n, budget, row = s["lengths"]
    at, there = _padded(row, n)
    new = torch.from_numpy(np.minimum(n, budget)).cuda()[:, None]
    pos = torch.where(there, s["pos"][at].long(), -1)
    last = pos.amax(-1, keepdim=True)
    safe = (pos >= 0) & ((pos < c["sinks"]) | (pos > last - c["recent"]))
    score = torch.where(pos >= 0, s["mass"][at], -1.0).masked_fill(safe, float("inf")).masked_fill(~there, float("-inf"))
    rank = torch.empty_like(at).scatter_(1, score.sort(dim=1, descending=True, stable=True).indices,
                                         torch.arange(at.shape[1], device="cuda").expand_as(at).contiguous())
    kept = rank < new
    i = torch.arange(at.shape[1], device="cuda")[None, :].expand_as(at)
    hole, moved = ~kept & (i < new), kept & (i >= new)
    src = torch.where(i < new, i, -1)
    src[hole] = i[moved]                                       # both in ascending order, as many of one as of the other in every cache
    live = i < new
    to, frm = at[live], (at - i)[live] + src[live]
    s["pos_out"][to], s["mass_out"][to], s["kept"][to] = s["pos"][frm], s["mass"][frm], src[live].int()
    to, frm = at[hole], at[moved]
    _bits(s["k"])[to], _bits(s["v"])[to] = _bits(s["k"])[frm], _bits(s["v"])[frm]
    return {"k": s["k"], "v": s["v"], "pos": s["pos_out"], "mass": s["mass_out"], "kept": s["kept"]}


# ---- the definitions in 64 bits


def exact(case, seed):
    global own
    before, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = before
    return {"rope": _exact_rope, "attend": _exact_attend, "evict": _exact_evict}[case["kind"]](s)


def _exact_rope(s):
    c = s["case"]
    H, G, d, r = c["heads"], c["kv_heads"], c["head_dim"], c["rot_dim"]
    x = s["qkv"].double().view(-1, H + 2 * G, d)
    weight = torch.cat([s["q_weight"].double().expand(H, d), s["k_weight"].double().expand(G, d)])
    y = x[:, :H + G]
    y = y / (y.pow(2).sum(-1, keepdim=True) / d + 1e-6).sqrt() * weight
    z = y.clone()
    for i in range(r // 2):
        a, b = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + r // 2)
        t = s["pos"].double() * s["inv_freq"][i]
        z[:, :, a] = y[:, :, a] * t.cos()[:, None] - y[:, :, b] * t.sin()[:, None]
        z[:, :, b] = y[:, :, a] * t.sin()[:, None] + y[:, :, b] * t.cos()[:, None]
    k, v = s["k_cache"].double(), s["v_cache"].double()
    k[s["out_rows"].long()], v[s["out_rows"].long()] = z[:, H:], x[:, H + G:]
    return {"q": z[:, :H], "k": k, "v": v}


def _exact_attend(s):
    c = s["case"]
    H, G, d = c["heads"], c["kv_heads"], c["head_dim"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(out.shape[:2], dtype=torch.float64, device="cuda")
    mass = s["mass"].double() if s["mass"] is not None else None
    for a, b, r, t in zip(*(x.tolist() for x in s["lengths"])):
        p = torch.arange(b - a, b, device="cuda") if s["q_pos"] is None else s["q_pos"][r:r + a].long()
        kp = torch.arange(b, device="cuda") if s["kv_pos"] is None else s["kv_pos"][t:t + b].long()
        blocked = (kp[None, :] > p[:, None]) | (kp[None, :] < 0)
        if c["window"]:
            blocked |= (kp[None, :] <= p[:, None] - c["window"]) & (kp[None, :] >= c["sinks"])
        for h in range(H):
            g = h * G // H
            l = s["q"][r:r + a, h].double() @ s["k"][t:t + b, g].double().T / d ** 0.5
            l[blocked] = float("-inf")
            z = torch.logsumexp(l, 1)
            w = torch.exp(l - torch.where(z == float("-inf"), 0.0, z)[:, None])
            out[r:r + a, h] = w @ s["v"][t:t + b, g].double()
            lse[r:r + a, h] = z
            if mass is not None:
                mass[t:t + b] += w.sum(0) / H
    return {"out": out, "lse": lse if s["lse"] is not None else None, "mass": mass}


def _exact_evict(s):
    c = s["case"]
    pos, mass = s["pos"].cpu().numpy(), s["mass"].double().cpu().numpy()
    out = {"k": s["k"].double(), "v": s["v"].double(), "pos": None, "mass": s["mass_out"].double(), "kept": None}
    for n, budget, row in zip(*(x.tolist() for x in s["lengths"])):
        p, m, new = pos[row:row + n], mass[row:row + n], min(n, budget)
        safe = (p < c["sinks"]) | (p > p.max() - c["recent"])
        best = np.lexsort((np.arange(n), -m, ~safe))[:new]     # protected rows first, then the heaviest, then the lower row
        holes = np.setdiff1d(np.arange(new), best)
        moved = np.sort(best[best >= new])
        src = np.arange(new)
        src[holes] = moved
        at = torch.from_numpy(row + src).cuda()
        out["mass"][row:row + new] = s["mass"].double()[at]
        out["k"][row:row + new], out["v"][row:row + new] = s["k"].double()[at], s["v"].double()[at]
    return out
