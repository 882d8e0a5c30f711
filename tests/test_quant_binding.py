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
