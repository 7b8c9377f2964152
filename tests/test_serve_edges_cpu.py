"""Host checks of the calls around the prune point at the ends of what they accept: no rows, no cache, scales and constants at the ends of 32 bits."""
import ctypes as C

import pytest

from test_serve_cpu import BAD, BF16, FP32, FP8, MB, ONE, OK, attention_call, eviction_call, rope_args, shim  # noqa: F401


@pytest.mark.parametrize("dtype", [BF16, FP32, FP8])
def test_no_rows_are_nothing_to_do_whatever_the_outputs_are(shim, dtype):  # noqa: F811
    """Tensors without rows have no address; the cache that they would go to has one."""
    for kw in (dict(q=None, k=None, v=None, pos=None), dict(q=None, k=None, v=None, q_out=None, pos=None, out_rows=None, kv_rows=1000),
               dict(k_out=None, v_out=None), dict(q=None, q_out=None, k=None, k_out=None, v=None, v_out=None)):
        assert shim.rope(dtype, 8, 4, 64, C.byref(rope_args(n_rows=0, **kw))) == OK
    for kw in (dict(rot_dim=80), dict(flags=4), dict(eps=-1.0), dict(kv_rows=-1)):       # (the numbers are looked at all the same)
        assert shim.rope(dtype, 8, 4, 64, C.byref(rope_args(n_rows=0, q=None, **kw))) == BAD


@pytest.mark.parametrize("want,scale", [(OK, 1e-38), (OK, 1.0), (OK, 2e38), (BAD, 1e-39), (BAD, 1e-300), (BAD, 3e38), (BAD, 1e300), (BAD, float("inf")),
                                        (BAD, float("nan"))])
def test_scales_that_32_bits_do_not_hold(shim, want, scale):  # noqa: F811
    for dtype in (BF16, FP32, FP8):
        assert attention_call(shim, ONE, dtype, scale=scale)[0] == want


def test_eviction_from_a_cache_without_rows(shim):  # noqa: F811
    none = dict(k=None, v=None, pos=None, mass=None, pos_out=None, mass_out=None)
    assert eviction_call(shim, [dict(n_kv=0, budget=5)], kv_rows=0, **none) == OK
    assert eviction_call(shim, [dict(n_kv=0, budget=5)] * 2, kv_rows=0, kv_len=6 * MB, kv_len_out=6 * MB, **none) == OK
    assert eviction_call(shim, [dict(n_kv=1, budget=5)], kv_rows=0, **none) == BAD
    for name in none:                                        # of a cache with rows everything is needed, whether the sequences have any or not
        assert eviction_call(shim, [dict(n_kv=0, budget=5)], **{name: None}) == BAD
