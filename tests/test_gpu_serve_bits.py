"""How exactly windowed attention's weights meet the values."""
import math

import pytest
import torch

import serve_util as R
from paper_2604_09244_b200.mvla import Seq
from test_gpu_serve import TYPES, context

pytestmark = pytest.mark.gpu


def levels(dtype, H, G, d, n_q, n_kv, key, value, scale):
    """A call whose queries all see the same logits, `scale` times `key[j]`; `value[j]` is all of row j's value.  Both are numbers of the type."""
    kept = TYPES[dtype]
    q = torch.zeros(n_q, H, d, device="cuda")
    q[..., 0] = 1
    k, v = torch.zeros(n_kv, G, d, device="cuda"), torch.zeros(n_kv, G, d, device="cuda")
    k[..., 0] = key[:, None]
    v[:] = value[:, None, None]
    assert bool((k.to(kept).float() == k).all()) and bool((v.to(kept).float() == v).all())
    pos = torch.full((n_q,), n_kv, dtype=torch.int32, device="cuda")
    return dict(seqs=[Seq(n_q=n_q, n_kv=n_kv)], q=q.to(kept), k=k.to(kept), v=v.to(kept), scale=scale, q_pos=pos)


def tolerance(r, d, meet):
    """As of any call: weights off by twice the logits' error, 2^-20 for powers of two and rescalings, 2^-24 a key for the sums, and by `meet` in
    the form in which they meet the values; then the rounding of the result."""
    own = (2 * R.logit_error(r["reach"], d) + 2.0 ** -20 + 2 * r["keys"] * 2.0 ** -24 + meet)[..., None] * r["weight"]
    return own + R.HALF[torch.bfloat16] * (r["out"].abs() + own) + 1e-30


@pytest.mark.parametrize("down", [18, 21, 23.5, 25.25, 27])
@pytest.mark.parametrize("heads", [(4, 1, 128), (2, 2, 64), (6, 2, 96), (2, 1, 256)])
@pytest.mark.parametrize("n_q", [1, 3, 70])
def test_faint_e4m3_keys_beside_strong_ones(n_q, heads, down):
    """One key in sixteen is 2^down times as strong as the others and has no value: what is left are the others' values.  fp16 weights are counted
    in units of 2^-7 of the reference (the largest weight, or less), so that one below fp16's normal numbers is off by 2^-25 2^-7 at most; sixteen
    such keys to a strong one, each with the value 448."""
    H, G, d = heads
    ctx = context("fp8", *heads)
    for n_kv in (64, 4001):
        hot = torch.arange(n_kv, device="cuda") % 16 == 5
        scale = down * math.log(2.0) / 16
        args = levels("fp8", H, G, d, n_q, n_kv, torch.where(hot, 16.0, 0.0), torch.where(hot, 0.0, 448.0), scale)
        r = R.attention(**args)[0]
        mass = torch.zeros(n_kv, device="cuda")
        for m in (None, mass):
            out = ctx.window_attention(**args, mass=m)
            err = (out.double() - r["out"]).abs()
            tol = tolerance(r, d, 2.0 ** -11) + 17 * 448 * 2.0 ** -32
            assert bool((err <= tol).all()), (n_kv, m is not None, float((err / tol).max()), float(out.float().mean()), float(r["out"].mean()))
    ctx.close()


@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 96), (16, 1, 160), (3, 3, 256), (4, 2, 64)])
@pytest.mark.parametrize("n_q", [1, 2, 4])
def test_weights_of_single_bf16_tokens(n_q, heads):
    """Values that cancel: half of the keys have weight 1 and value 1, half weight e^(-2^-9) and value -1.  The smaller weight lies between two bf16
    numbers 2^-8 apart; single tokens (at most 16 query rows to a key head) keep what rounding leaves of a weight, so that weights are
    off by 2^-16 at most, whichever form the call takes: with accumulated weights or without."""
    H, G, d = heads
    if n_q * H // G > 16:
        pytest.skip("no single token")
    ctx = context("bf16", *heads)
    for n_kv in (64, 1000, 20012):
        odd = torch.arange(n_kv, device="cuda") % 2 == 1
        args = levels("bf16", H, G, d, n_q, n_kv, torch.where(odd, -2.0 ** -9, 0.0), torch.where(odd, -1.0, 1.0), 1.0)
        r = R.attention(**args)[0]
        mass = torch.zeros(n_kv, device="cuda")
        for m in (None, mass):
            out = ctx.window_attention(**args, mass=m)
            err, tol = (out.double() - r["out"]).abs(), tolerance(r, d, 2.0 ** -16)
            assert bool((err <= tol).all()), (n_kv, m is not None, float((err / tol).max()))
    ctx.close()


@pytest.mark.parametrize("mass", [False, True])
def test_weights_of_a_single_bf16_token_beside_a_block(mass):
    """The same token in a batch with a block of queries, and with a much longer sequence: as exact as alone."""
    H, G, d, n_kv = 8, 2, 128, 700
    ctx = context("bf16", H, G, d)
    odd = torch.arange(n_kv, device="cuda") % 2 == 1
    one = levels("bf16", H, G, d, 1, n_kv, torch.where(odd, -2.0 ** -9, 0.0), torch.where(odd, -1.0, 1.0), 1.0)
    r = R.attention(**one)[0]
    for n_q, more in ((200, 300), (1, 30000), (5, 700)):
        q = torch.cat([one["q"], one["q"][:1].expand(n_q, -1, -1)])
        k, v = (torch.cat([one[x], torch.zeros(more, G, d, device="cuda").bfloat16()]) for x in ("k", "v"))
        seqs = [Seq(n_q=1, n_kv=n_kv), Seq(q_row=1, n_q=n_q, kv_row=n_kv, n_kv=more)]
        pos = torch.full((1 + n_q,), n_kv, dtype=torch.int32, device="cuda")
        out = ctx.window_attention(seqs, q, k, v, scale=1.0, q_pos=pos, mass=torch.zeros(n_kv + more, device="cuda") if mass else None)
        err, tol = (out[:1].double() - r["out"]).abs(), tolerance(r, d, 2.0 ** -16)
        assert bool((err <= tol).all()), (n_q, more, float((err / tol).max()))
    ctx.close()
