"""The calls around the prune point in 64 bits, written from their definitions, with how far a result may be off."""
import torch

# Half a step of each type, relative to the value.
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float8_e4m3fn: 2.0 ** -4}
WIDE = {torch.float32: torch.float32, torch.bfloat16: torch.bfloat16, torch.float8_e4m3fn: torch.bfloat16}


def rope(x, pos, inv_freq, weight, norm, eps, interleaved):
    """(z, size): rotated rows, and for every element |y_a| + |y_b| of its pair, in 64 bits on the tensor's device."""
    y = x.double()
    if norm:
        y = y / (y.pow(2).mean(-1, keepdim=True) + eps).sqrt()
        if weight is not None:
            y = y * weight.double()
    r = 0 if inv_freq is None else 2 * inv_freq.numel()
    z, size = y.clone(), y.abs().clone()
    if r:
        t = pos.double()[:, None] * inv_freq[None, :]
        c, s = t.cos()[:, None, :], t.sin()[:, None, :]
        i = torch.arange(r // 2, device=x.device)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + r // 2)
        z[..., a], z[..., b] = y[..., a] * c - y[..., b] * s, y[..., b] * c + y[..., a] * s
        size[..., a] = size[..., b] = y[..., a].abs() + y[..., b].abs()
    return z, size


def rope_tolerance(z, size, dtype, far=0):
    """The kernel's own arithmetic: a sum of up to 256 squares in a tree (relative 2^-24 per level and product, halved by the root),
    division, root and two products (four half steps), the cosine and sine (2 units of 2^-24 each, absolute), two products and
    a sum: under 24 half steps of the pair's size.  The angle itself, in turns and in 64 bits, is off by three roundings of the
    position's turns (far / (2 pi) at most) on either side.  Then one rounding to the kept type (of e4m3's smallest values half of 2^-9)."""
    own = (24 * 2.0 ** -24 + 6 * 2.0 ** -53 * far) * size
    return own + HALF[dtype] * (z.abs() + own) + (2.0 ** -10 if dtype == torch.float8_e4m3fn else 1e-37)


def attention(seqs, q, k, v, window=None, n_sink=0, scale=0.0, q_pos=None, kv_pos=None, kv_len=None):
    """Per sequence: dict of out, lse, mass (increment), and what their tolerances need, in 64 bits."""
    H, d = q.shape[1], q.shape[2]
    G = k.shape[1]
    dev = q.device
    scale = scale or d ** -0.5
    found = []
    for b, s in enumerate(seqs):
        n = s.n_kv if kv_len is None else max(0, min(int(kv_len[b]), s.n_kv))
        p = q_pos[s.q_row:s.q_row + s.n_q].long() if q_pos is not None else torch.arange(s.n_q, device=dev) + (n - s.n_q)
        c = kv_pos[s.kv_row:s.kv_row + n].long() if kv_pos is not None else torch.arange(n, device=dev)
        vis = (c[None] >= 0) & (c[None] <= p[:, None])
        if window is not None:
            vis = vis & ((p[:, None] - c[None] < window) | (c[None] < n_sink))
        any_vis = vis.any(1)
        used = vis.any(0)
        qd = q[s.q_row:s.q_row + s.n_q].double()
        kd = torch.where(used[:, None, None], k[s.kv_row:s.kv_row + n].double(), 0.0)
        vd = torch.where(used[:, None, None], v[s.kv_row:s.kv_row + n].double(), 0.0)
        kd, vd = kd.repeat_interleave(H // G, 1), vd.repeat_interleave(H // G, 1)
        l = torch.einsum("ihd,jhd->hij", qd, kd) * scale
        reach = torch.einsum("ihd,jhd->hij", qd.abs(), kd.abs()).mul(scale).masked_fill(~vis[None], 0.0)
        reach = reach.amax(-1) if n else torch.zeros(H, s.n_q, device=dev, dtype=torch.float64)          # [H, n_q]
        l = l.masked_fill(~vis[None], float("-inf"))
        lse = torch.logsumexp(l, -1) if n else torch.full((H, s.n_q), float("-inf"), device=dev, dtype=torch.float64)
        w = torch.exp(l - torch.where(any_vis[None], lse, 0.0)[..., None])
        found.append({"out": torch.einsum("hij,jhd->ihd", w, vd), "weight": torch.einsum("hij,jhd->ihd", w, vd.abs()), "lse": lse.T,
                      "mass": w.sum((0, 1)) / H, "reach": reach.T, "n": n, "rows": any_vis, "keys": int(vis.sum(1).max()) if n and s.n_q else 0})
    return found


def logit_error(reach, d):
    """How far a logit may be off: a dot product of d terms in 32 bits, in any order and with sums that a tensor core may cut off
    instead of rounding (twice 2^-24 a step), its scale, the difference to the running maximum (both as large as the logits): absolute."""
    return (2 * d + 16) * 2.0 ** -24 * reach + 2.0 ** -22


def attention_tolerance(r, d, dtype):
    """out: weights off by twice the logits' error (numerator and denominator), by 2^-21 for the power of two, by the rescalings and sums
    (2^-24 a key, at most), and by half a step of the type in which they meet the values; then the rounding of the result.
    (fp16 weights below its smallest normal number, 2^-14, are off by 2^-25 of the largest weight each: with `keys` of them against one,
    keys 2^-25 of the largest value.)"""
    meet = {torch.float32: 0.0, torch.bfloat16: HALF[torch.bfloat16], torch.float8_e4m3fn: HALF[torch.float16]}[dtype]
    per_weight = 2 * logit_error(r["reach"], d) + 2.0 ** -20 + 2 * r["keys"] * 2.0 ** -24 + meet
    own = per_weight[..., None] * r["weight"]
    if dtype == torch.float8_e4m3fn:
        own = own + r["keys"] * 2.0 ** -25 * 448.0 / 64
    return own + HALF[WIDE[dtype]] * (r["out"].abs() + own) + 1e-30


def mass_tolerance(r, d, n_q, H, before):
    rel = 2 * float(logit_error(r["reach"].max(), d)) + 2.0 ** -20 + (2 * r["keys"] + n_q + H) * 2.0 ** -24 if r["reach"].numel() else 0.0
    return rel * r["mass"] + 2.0 ** -24 * (before.abs() + r["mass"]) * 2 + 1e-30


def evict(seqs, pos, mass, n_sink, n_recent, kv_len=None):
    """Per sequence the rows (relative) that are row 0, 1, ... afterwards."""
    found = []
    for b, s in enumerate(seqs):
        n = s.n_kv if kv_len is None else max(0, min(int(kv_len[b]), s.n_kv))
        m = min(n, s.budget)
        p = pos[s.kv_row:s.kv_row + n].tolist()
        w = mass[s.kv_row:s.kv_row + n].tolist()
        last = max(p, default=-1)

        def rank(j):
            if p[j] < 0:
                return (3, 0.0, j)
            if p[j] < n_sink or last - p[j] < n_recent:
                return (0, 0.0, j)
            return (2, 0.0, j) if w[j] != w[j] else (1, -w[j], j)

        kept = sorted(sorted(range(n), key=rank)[:m])
        stay = set(kept)
        holes = [j for j in range(m) if j not in stay]
        src = list(range(m))
        for hole, row in zip(holes, [j for j in kept if j >= m]):
            src[hole] = row
        found.append(src)
    return found
