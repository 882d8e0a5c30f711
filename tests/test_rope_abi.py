"""Which calls of the rotation are taken and which refused, before any launch (no GPU needed)."""

import ctypes
import random

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


def rows_of(first, stride, extent):
    return sorted(first + b * stride[0] + h * stride[1] + r * stride[2]
                  for b in range(extent[0]) for h in range(extent[1]) for r in range(extent[2]))


def overlap(a, b, nbytes):
    """(library's verdict, every row against every row) for operands (first byte, strides, extents)."""
    fn = rk.lib().reskv_internal_rows_overlap
    fn.restype, fn.argtypes = ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64]
    x, y = ((ctypes.c_int64 * 7)(first, *stride, *extent) for first, stride, extent in (a, b))
    ra, rb = rows_of(*a), rows_of(*b)
    return fn(x, y, nbytes), int(any(abs(p - q) < nbytes for p in ra for q in rb))


@pytest.mark.parametrize("seed", range(8))
def test_overlap_of_rows_is_exact(seed):
    """Against every pair of rows: operands with strides of their own, of each other, broadcast, and slices of one
    buffer."""
    rng = random.Random(seed)
    said = set()
    for _ in range(400):
        n = rng.choice([16, 64, 128])
        extent = [rng.randint(1, 3), rng.randint(1, 5), rng.randint(1, 5)]
        order, stride, span = rng.sample(range(3), 3), [0, 0, 0], n * rng.randint(1, 3)
        for i in order:  # each passes what the ones before it span
            stride[i] = span + 16 * rng.choice([0, 0, 1, 5, 40])
            span = stride[i] * extent[i]
        a = (1 << 20, tuple(stride), tuple(extent))
        heads = rng.choice([extent[1], 1, rng.randint(1, 6)])
        other = rng.choice([stride, [stride[0], 2 * stride[1], stride[2]], [stride[0], 0, stride[2]],
                            [16 * rng.randint(0, 60) for _ in range(3)]])
        b = ((1 << 20) + 16 * rng.randint(-span // 16 - 8, span // 16 + 8), tuple(other), (extent[0], heads, extent[2]))
        got, want = overlap(a, b, n)
        assert got == want, (a, b, n)
        said.add(got)
    assert said == {0, 1}


def test_overlap_of_slices_at_full_size():
    """Parts of a fused projection of 65536 tokens, in turns of the same and of another order."""
    d, heads, tokens = 256, 48, 65536
    token_major = (0, d, heads * d)
    fn = rk.lib().reskv_internal_rows_overlap
    fn.restype, fn.argtypes = ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64]

    def verdict(a, b):
        return fn(*((ctypes.c_int64 * 7)(x[0], *x[1], *x[2]) for x in (a, b)), d)

    q = ((1 << 32), token_major, (1, 32, tokens))
    for first, want in ((32, 0), (31, 1), (40, 0), (0, 1)):
        assert verdict(q, ((1 << 32) + first * d, token_major, (1, 8, tokens))) == want
    assert verdict(q, ((1 << 32) + 32 * d, (0, 2 * d, heads * d), (1, 8, tokens))) == 0  # every other head
    assert verdict(q, ((1 << 32) + 31 * d, (0, 2 * d, heads * d), (1, 8, tokens))) == 1
    head_major = (0, tokens * d, d)
    assert verdict(q, ((1 << 32) + heads * tokens * d, head_major, (1, 32, tokens))) == 0
    assert verdict(q, ((1 << 32) + 48 * d, head_major, (1, 32, tokens))) == 1


ROWS = (5120, 640, 128)  # of q [2, 8, 5, 128]
KROWS = (1280, 640, 128)


@pytest.mark.parametrize("kw", [
    dict(q=(P, ROWS), q_out=(2 * P, ROWS), k=(3 * P, KROWS), k_out=(P, KROWS)),             # keys over the queries
    dict(q=(P, ROWS), q_out=(2 * P, ROWS), k=(2 * P + 256, KROWS), k_out=(3 * P, KROWS)),   # queries over the keys
    dict(q=(P, ROWS), q_out=(2 * P, ROWS), k=(3 * P, KROWS), k_out=(2 * P, KROWS)),         # both into one place
    dict(q=(P, ROWS), q_out=(P, ROWS), k=(P, KROWS), k_out=(P, KROWS)),                     # in place, both the same
    # a fused projection of 12 heads, keys one head early
    dict(q=(P, (7680, 128, 1536)), q_out=(P, (7680, 128, 1536)), k=(P + 7 * 256, (7680, 128, 1536)),
         k_out=(P + 7 * 256, (7680, 128, 1536)))])
def test_queries_and_keys_overlap(kw):
    """Queries and keys are rotated side by side: an output over the other's input or output has no order."""
    assert call(shape(), 5, **kw) == 1
    assert "overlap" in rk.last_error()


def test_overlap_search_ends():
    """Strides without a common order, apart by a few bytes: given up after a bounded search, never called apart
    where rows meet."""
    fn = rk.lib().reskv_internal_rows_overlap
    fn.restype, fn.argtypes = ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64]
    verdicts = set()
    for shift in range(0, 4096, 16):
        a = (1 << 32, (0, 4096 * 10007, 4096 * 9973), (1, 2000, 2000))
        b = ((1 << 32) + (1 << 34) + shift, (0, 4096 * 9941, 4096 * 10037), (1, 2000, 2000))
        verdicts.add((shift < 64 or shift > 4096 - 64,
                      fn(*((ctypes.c_int64 * 7)(x[0], *x[1], *x[2]) for x in (a, b)), 64)))
    assert {v for near, v in verdicts if not near} == {0}       # by what all strides are multiples of
    assert {v for near, v in verdicts if near} <= {1, 2}
    a = (1 << 32, (0, 16 * 10007, 16 * 9973), (1, 20000, 20000))
    b = ((1 << 32) + (1 << 31) + 8, (0, 32 * 4970, 32 * 5018), (1, 20000, 20000))
    assert fn(*((ctypes.c_int64 * 7)(x[0], *x[1], *x[2]) for x in (a, b)), 16) in (1, 2)
