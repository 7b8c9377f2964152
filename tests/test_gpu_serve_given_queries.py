"""Windowed attention where positions of the queries are given and cached rows are counted, up to the last position of the type."""
import pytest
import torch

from test_gpu_serve import attend_case, check_attention, context

pytestmark = pytest.mark.gpu

TOP = 2 ** 31 - 1


def given(args, kind, seed):
    """Positions for the queries of a call whose cached rows are counted."""
    gen = torch.Generator("cuda").manual_seed(seed)
    pos = torch.full((args["q"].shape[0],), -1, dtype=torch.int32, device="cuda")
    for s in args["seqs"]:
        p = torch.randint(0, 2 * s.n_kv + 2, (s.n_q,), generator=gen, device="cuda", dtype=torch.int32)
        if kind == "last":
            p[:] = TOP
        elif kind == "beside":                               # the last position, and positions of no row, next to ordinary ones
            p[::3] = TOP
            p[1::5] = -1 - p[1::5]
            p[2::7] = -(2 ** 31)
        pos[s.q_row:s.q_row + s.n_q] = p
    return dict(args, q_pos=pos)


@pytest.mark.parametrize("kind", ["last", "beside", "scattered"])
@pytest.mark.parametrize("n_q", [1, 3, 50, 300])
@pytest.mark.parametrize("dtype", ["bf16", "fp32", "fp8"])
def test_given_positions_of_queries_over_counted_rows(dtype, n_q, kind):
    for heads in ((4, 2, 64), (8, 2, 128)):
        ctx = context(dtype, *heads)
        for i, (window, sinks) in enumerate(((None, 0), (30, 2), (TOP - 1, 0), (1, 0), (7, TOP))):
            for mass in (True, False):
                args, weights, kept = attend_case(dtype, *heads, [n_q, n_q], [200, 71], window, sinks, "count", seed=i, mass=mass)
                check_attention(ctx, given(args, kind, i), weights, kept)
        ctx.close()


@pytest.mark.parametrize("dtype,n_q", [("bf16", 1), ("bf16", 40), ("fp32", 1), ("fp32", 40), ("fp8", 1), ("fp8", 40)])
def test_given_positions_over_rows_in_parts(dtype, n_q):
    """Long enough for the keys to be cut into parts."""
    ctx = context(dtype, 4, 1, 128)
    for kind in ("last", "beside", "scattered"):
        for mass in (True, False):
            args, weights, kept = attend_case(dtype, 4, 1, 128, [n_q, 1], [9000, 300], 4000, 6, "count", seed=2, mass=mass)
            for window in (None, 4000):
                check_attention(ctx, dict(given(args, kind, 5), window=window), weights, kept)
    ctx.close()
