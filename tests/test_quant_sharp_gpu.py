"""Decode over 4-bit caches where one key has all the weight: its value comes out and p_max is 1, however large its
logit and however coarsely 32 bits hold it."""

import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2607_29591_amd import reskv as rk
from tests.test_quant_decode_gpu import Case, dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("C,split", [(300, 1), (3000, 6)])
@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("e", [8, 12, 17, 20, 23, 26, 28, 29, 30, 31, 34])
def test_one_key_with_all_the_weight(dtype, d, e, C, split):
    """Logits of about 2^e; every other main key is 0, e^-2^e beside it. Units that are full of main slots (at 100,
    and at 1700 of a split head), and one with residual slots and the end in it (at 200)."""
    H, G = 3, 2
    r = np.array([[0, 64, 130]])
    n = np.array([[C - 1, C - 64, 100]])
    c = Case(e, dtype, d, 1, H, G, C, 130, r, n)
    assert rk.lib().reskv_internal_quant_parts(ctypes.byref(c.shape)) == split
    q = np.abs(c.rng.normal(size=(1, H * G, d))) + 0.5
    c.q = dev(q, dtype)
    kc, vc = torch.zeros(1, H, C, d, dtype=c.q.dtype, device="cuda"), dev(c.V, dtype)
    at = [100, 1700 if split > 1 else 150, 200]
    for h in range(H):
        kc[0, h, at[h]] = 2.0 ** (e - round(math.log2(1.3 * math.sqrt(d))))  # logit: sum q k / sqrt(d)
    rk.reskv_pack_quant(c.shape, kc, vc, c.res_len, c.main_len, c.cache)
    out, lse_main, _, gate = c.decode(dict(tau_scalar=0.9, alpha=12.0))
    want = np.stack([c.V[0, h, at[h]] for h in range(H)]).repeat(G, 0)
    got = out[0].double().cpu().numpy()
    # the probability is 1, exact in bf16; the denominator's other terms vanish; a few roundings of 2^-24
    assert (np.abs(got - want) <= 8 * 2.0 ** -24 * np.abs(want)).all()
    # sigmoid(12 (0.9 - 1)) in 32 bits: the difference is off by 2^-25, the product and the exponential by a few 2^-24
    g = 1 / (1 + math.exp(1.2))
    assert (np.abs(gate.double().cpu().numpy() - g) <= 16 * 2.0 ** -24).all()
    logit = (c.q.double().cpu().numpy() * float(kc.max())).sum(-1) / math.sqrt(d)
    # a sum of 3 d exact products in 32 bits, scaled
    assert (np.abs(lse_main.double().cpu().numpy() - logit) <= (3 * d + 8) * 2.0 ** -24 * logit).all()
