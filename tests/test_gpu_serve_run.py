"""The calls around the prune point as they are used, one behind the other: a prune step, projections of the rows that it keeps, their norms and
rotation into a cache, the prefill's attention with accumulated weights, eviction, then single tokens.  Every step is held against the 64-bit
reference of its own inputs."""
import pytest
import torch

import serve_util as R
from paper_2604_09244_b200 import mvla
from paper_2604_09244_b200 import workloads as W
from paper_2604_09244_b200.mvla import Seq
from parity_util import device_tensors
from test_gpu_serve import bits

pytestmark = pytest.mark.gpu

WINDOW, SINKS, RECENT, BUDGET, SPARE = 40, 3, 8, 50, 4


class Run:
    """Caches of two requests of a pruned frame, with one row over the budget for the token of the next step."""

    def __init__(self, dtype, G):
        self.wl = wl = W.small_workload(5, batch=2, D=512, H=8, d=64, dtype=dtype, n_txt=(9, 17), n_2d=(90, 130), n_3d=(80, 60), n_kv_heads=G)
        self.H, self.G, self.d = wl.n_heads, G or wl.n_heads, wl.head_dim
        self.ctx = mvla.context_for(wl)
        dev = device_tensors(wl)
        self.kept_type, self.wide = dev["k"].dtype, dev["hidden"].dtype
        o = self.ctx.prune_step(0, wl.samples, wl.mode, dev["q"], dev["k"], dev["v"], dev["hidden"])
        at = o.out_offsets.tolist()
        self.n = [b - a for a, b in zip(at, at[1:])]
        assert min(self.n) > BUDGET + 1
        self.hidden, self.pos = o.out_hidden[:at[-1]], o.kept_idx[:at[-1]]
        gen = torch.Generator("cuda").manual_seed(3)
        self.w = (torch.randn(wl.d_model, (self.H + 2 * self.G) * self.d, generator=gen, device="cuda") * wl.d_model ** -0.5).to(self.wide)
        self.wq, self.wk = ((1 + 0.2 * torch.randn(self.d, generator=gen, device="cuda")).to(self.wide) for _ in range(2))
        self.freq = 10000.0 ** (-torch.arange(0, self.d, 2, device="cuda", dtype=torch.float64) / self.d)
        self.tokens = torch.randn(6, 2, wl.d_model, generator=gen, device="cuda").to(self.wide)
        self.base = [2, 2 + self.n[0] + SPARE]
        rows = self.base[1] + self.n[1] + SPARE
        self.k, self.v = (torch.full((rows, self.G, self.d), float("nan"), device="cuda").to(self.kept_type) for _ in range(2))
        self.kv_pos = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
        self.mass = torch.zeros(rows, device="cuda")

    def rows_of(self, hidden, pos, to):
        """Projections, norms and rotation of rows, which become rows `to` of the caches; the rotated queries."""
        q, k, v = (x.unflatten(1, (-1, self.d)) for x in (hidden @ self.w).split([self.H * self.d, self.G * self.d, self.G * self.d], 1))
        q_out, _, _ = self.ctx.qk_norm_rope(q, k, pos, self.freq, v=v, q_weight=self.wq, k_weight=self.wk, k_out=self.k, v_out=self.v, out_rows=to)
        self.kv_pos.index_copy_(0, to.long(), pos)
        return q, k, v, q_out

    def attend(self, seqs, q, q_pos, kv_len=None):
        return self.ctx.window_attention(seqs, q, self.k, self.v, window=WINDOW, n_sink=SINKS, q_pos=q_pos, kv_pos=self.kv_pos, kv_len=kv_len,
                                         mass=self.mass)

    def evict(self, lens, kv_len=None, kv_len_out=None):
        self.ctx.cache_evict([Seq(kv_row=b, n_kv=n, budget=BUDGET) for b, n in zip(self.base, lens)], self.k, self.v, self.kv_pos, self.mass,
                             n_sink=SINKS, n_recent=RECENT, kv_len=kv_len, kv_len_out=kv_len_out)

    def check_rows(self, q, k, v, q_out, pos, to):
        for x, w, got in ((q, self.wq, q_out), (k, self.wk, self.k[to.long()])):
            z, size = R.rope(x, pos, self.freq, w, True, 1e-6, False)
            assert bool(((got.double() - z).abs() <= R.rope_tolerance(z, size, self.kept_type, 1000)).all())
        assert torch.equal(bits(self.v[to.long()]), bits(v.to(self.kept_type)))

    def check_attention(self, seqs, q, q_pos, out, before):
        refs = R.attention(seqs, q, self.k, self.v, WINDOW, SINKS, 0.0, q_pos, self.kv_pos)
        for s, r in zip(seqs, refs):
            assert bool(r["rows"].all())                     # a token sees itself
            o = out[s.q_row:s.q_row + s.n_q].double()
            assert bool(((o - r["out"]).abs() <= R.attention_tolerance(r, self.d, self.kept_type)).all())
            c = slice(s.kv_row, s.kv_row + s.n_kv)
            grown = self.mass[c].double() - before[c].double()
            assert bool(((grown - r["mass"]).abs() <= R.mass_tolerance(r, self.d, s.n_q, self.H, before[c].double())).all())
            assert abs(float(grown.sum()) - s.n_q) < 1e-3 * s.n_q       # the weights of a query sum to one

    def check_evict(self, lens, before):
        k, v, pos, mass = before
        want = R.evict([Seq(kv_row=b, n_kv=n, budget=BUDGET) for b, n in zip(self.base, lens)], pos.cpu(), mass.cpu(), SINKS, RECENT)
        for b, src in zip(self.base, want):
            at, rows = b + torch.tensor(src, device="cuda"), slice(b, b + BUDGET)
            assert len(src) == BUDGET
            assert torch.equal(bits(self.k)[rows], bits(k)[at]) and torch.equal(bits(self.v)[rows], bits(v)[at])
            assert torch.equal(self.kv_pos[rows], pos[at]) and torch.equal(self.mass[rows], mass[at])

    def state(self):
        return [x.clone() for x in (self.k, self.v, self.kv_pos, self.mass)]

    def prefill(self):
        to = torch.cat([torch.arange(b, b + n) for b, n in zip(self.base, self.n)]).to("cuda", torch.int32)
        rotated = self.rows_of(self.hidden, self.pos, to)
        self.check_rows(*rotated, self.pos, to)
        seqs = [Seq(q_row=a, n_q=n, kv_row=b, n_kv=n) for a, n, b in zip((0, self.n[0]), self.n, self.base)]
        before = self.mass.clone()
        out = self.attend(seqs, rotated[3], self.pos)
        self.check_attention(seqs, rotated[3], self.pos, out, before)
        old = self.state()
        self.evict(self.n)
        self.check_evict(self.n, old)
        self.to = torch.tensor([b + BUDGET for b in self.base], dtype=torch.int32, device="cuda")
        self.seqs = [Seq(q_row=i, n_q=1, kv_row=b, n_kv=BUDGET + 1) for i, b in enumerate(self.base)]
        self.next = [int(self.pos[self.n[0] - 1]) + 1, int(self.pos[-1]) + 1]

    def positions(self, step):
        return torch.tensor([p + step for p in self.next], dtype=torch.int32, device="cuda")

    def token(self, hidden, pos, check):
        rotated = self.rows_of(hidden, pos, self.to)
        if check:
            self.check_rows(*rotated, pos, self.to)
            before = self.mass.clone()
        if check:
            before[self.to.long()] = 0
        self.mass.index_fill_(0, self.to.long(), 0.0)        # the new row has no weight yet
        out = self.attend(self.seqs, rotated[3], pos)
        if check:
            self.check_attention(self.seqs, rotated[3], pos, out, before)
            old = self.state()
        self.evict([BUDGET + 1] * 2)
        if check:
            self.check_evict([BUDGET + 1] * 2, old)
        return out


@pytest.mark.parametrize("dtype,G", [("bf16", 0), ("bf16", 2), ("fp8", 2), ("fp32", 0)])
def test_pruned_frame_to_tokens(dtype, G):
    run = Run(dtype, G)
    run.prefill()
    start = run.state()
    outs = [run.token(run.tokens[i], run.positions(i), True) for i in range(len(run.tokens))]
    end = run.state()
    # the same tokens with the whole step in one graph
    for x, y in zip((run.k, run.v, run.kv_pos, run.mass), start):
        bits(x).copy_(bits(y))
    hidden, pos = run.tokens[0].clone(), run.positions(0)
    warm = torch.cuda.Stream()
    with torch.cuda.stream(warm):
        hidden @ run.w                               # (the library's own workspace, outside the capture)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run.token(hidden, pos, False)
    for i, want in enumerate(outs):
        hidden.copy_(run.tokens[i])
        pos.copy_(run.positions(i))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    for x, y in zip((run.k, run.v, run.kv_pos, run.mass), end):
        for b in run.base:
            assert torch.equal(bits(x)[b:b + BUDGET], bits(y)[b:b + BUDGET])
    run.ctx.close()
