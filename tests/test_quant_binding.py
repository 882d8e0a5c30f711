"""What the binding keeps of a call's arguments (no GPU needed)."""

import gc
import weakref

import torch

from paper_2607_29591_amd import reskv as rk

B, Hq = 2, 8


def test_thresholds_live_as_long_as_their_gate():
    tau = torch.zeros(B, Hq)
    gate, gone = rk.make_gate(tau=tau), weakref.ref(tau)
    del tau
    gc.collect()
    assert gone() is not None and gate.tau == gone().data_ptr()
    del gate
    gc.collect()
    assert gone() is None
