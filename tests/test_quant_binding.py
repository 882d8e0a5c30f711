"""What the binding of the rotation and the 4-bit caches refuses before it takes a pointer (no GPU needed: type and
size are looked at before the device)."""

import gc
import weakref

import pytest
import torch

from paper_2607_29591_amd import reskv as rk

B, Hq, H, d, C = 2, 8, 2, 128, 640


def shape():
    return rk.make_shape(B, Hq, H, d, "bf16", C, 64)


def decode(gate):
    s = shape()
    lens = torch.zeros(B * H, dtype=torch.int32)
    rk.reskv_decode_attn_quant(s, gate, torch.zeros(B, Hq, d, dtype=torch.bfloat16),
                               torch.zeros(rk.reskv_quant_cache_size(s), dtype=torch.uint8), torch.zeros(B, H, 64), lens,
                               lens, torch.zeros(B, Hq, d), torch.zeros(4, dtype=torch.uint8))


def test_thresholds_live_as_long_as_their_gate():
    tau = torch.zeros(B, Hq)
    gate, gone = rk.make_gate(tau=tau), weakref.ref(tau)
    del tau
    gc.collect()
    assert gone() is not None and gate.tau == gone().data_ptr()
    del gate
    gc.collect()
    assert gone() is None


@pytest.mark.parametrize("tau,match", [
    (torch.zeros(B, Hq, dtype=torch.bfloat16), "tau must be torch.float32"),
    (torch.zeros(B, Hq, dtype=torch.float64), "tau must be torch.float32"),
    (torch.zeros(B, Hq - 1), "tau must have 16 elements"), (torch.zeros(1), "tau must have 16 elements"),
    (torch.zeros(B, Hq), "tau must be on the current GPU")])
def test_thresholds_are_checked_as_every_tensor_is(tau, match):
    with pytest.raises(ValueError, match=match):
        decode(rk.make_gate(tau=tau))


def rows(*size):
    return torch.zeros(*size, dtype=torch.bfloat16)


@pytest.mark.parametrize("k,v", [((B, 5, H, d), (B, 5, H, d)), ((B, H, 5, d), (B, 5, H, d)), ((B, H, 5, d), (B, H, d, 5)),
                                 ((H * 5, 1, B, d), (B, H, 5, d))])
def test_rows_of_another_order_are_refused(k, v):
    """Tensors of the right number of elements whose heads and tokens lie in another order than [B, Hkv, n, d]."""
    s, lens = shape(), torch.zeros(B * H, dtype=torch.int32)
    cache = torch.zeros(rk.reskv_quant_cache_size(s), dtype=torch.uint8)
    with pytest.raises(ValueError, match=r"must be \[2, 2, \d+, 128\]"):
        rk.reskv_append_kv_quant(s, rows(*k), rows(*v), cache, lens, lens)
    with pytest.raises(ValueError, match=r"must be \[2, 2, \d+, 128\]"):
        rk.reskv_unpack_quant(s, cache, lens, lens, rows(*k), rows(*v))
    with pytest.raises(ValueError, match=r"must be \[2, 2, 640, 128\]"):
        rk.reskv_pack_quant(s, *(rows(*(C if x == 5 else x for x in t)) for t in (k, v)), lens, lens, cache)


def test_positions_of_another_order_are_refused():
    s, lens = shape(), torch.zeros(B * H, dtype=torch.int32)
    with pytest.raises(ValueError, match=r"positions must be \[2, 5\]"):
        rk.reskv_append_kv_quant(s, rows(B, H, 5, d), rows(B, H, 5, d),
                                 torch.zeros(rk.reskv_quant_cache_size(s), dtype=torch.uint8), lens, lens,
                                 rope=rk.make_rope(64), positions=torch.zeros(5, B, dtype=torch.int32))
