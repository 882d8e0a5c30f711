"""Which calls of the rotation are taken and which refused, before any launch (no GPU needed)."""

import ctypes

import pytest

from paper_2607_29591_amd import reskv as rk

P = 1 << 32  # an address that no call here follows


def shape(**kw):
    return rk.make_shape(**dict(dict(batch=2, num_q_heads=8, num_kv_heads=2, head_dim=128, dtype="bf16", slot_cap=1,
                                     res_cap=1), **kw))


def call(s, n, q=None, q_out=None, k=None, k_out=None):
    """Status of a call; each operand is (address, (batch, head, row) strides in elements)."""
    at = []
    for x in (q, q_out, k, k_out):
        at += [None, None] if x is None else [x[0], ctypes.byref(rk.Rows(*x[1]))]
    return rk.lib().reskv_rope(ctypes.byref(s), ctypes.byref(rk.Rope(64, 0, 1.0, P)), n, P, None, *at, None)


@pytest.mark.parametrize("kw", [dict(slot_cap=0), dict(res_cap=0), dict(slot_cap=-1, res_cap=-1),
                                dict(batch=64, slot_cap=2 ** 31 - 1)])
def test_cache_sizes_are_not_used(kw):
    """slot_cap and res_cap say nothing about a rotation, whatever they hold."""
    assert call(shape(**kw), 0) == 0


@pytest.mark.parametrize("hq,hkv,code", [(2 ** 30, 2 ** 30, 2), (2 ** 31 - 1, 2 ** 31 - 1, 2), (2 ** 30, 2 ** 26, 2),
                                         (2 ** 25 + 1, 2 ** 25 + 1, 2)])
def test_more_heads_than_a_launch_indexes(hq, hkv, code):
    """Head numbers are 32-bit, and a wave looks a few heads past its last: 2^26 heads in all are taken. The rows
    here lie apart from each other, so nothing else refuses the call."""
    hq -= hq % hkv
    s = shape(batch=1, num_q_heads=hq, num_kv_heads=hkv, head_dim=64)
    at = (2 ** 48, 64, 64)
    assert call(s, 1, q=(P, at), q_out=(P, at)) == code
    assert "heads" in rk.last_error()
