"""fp32 numbers one step beside the borders between two 4-bit values, and beside the borders of the scale rule, at the
scales' ends too, where the numbers are subnormal: bytes and values are the definition's."""

import numpy as np
import pytest
import torch

from paper_2607_29591_amd import reskv as rk
from tests import quant_ref as ref
from tests.test_quant_gpu import filled, host, i32

pytestmark = pytest.mark.gpu


def rows():
    groups = []
    for k in (-125, -124, -100, -1, 0, 7, 100, 124, 125):
        border = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.5, 1.0, 6.0]) * 2.0 ** k
        x = border.astype(np.float32)
        x = np.concatenate([np.nextafter(x, np.float32(0)), x, np.nextafter(x, np.float32(np.inf))])
        for top in (4.0, 6.0, 7.0):
            for sign in (1, -1):
                groups.append(np.concatenate([[np.float32(top * 2.0 ** k)], sign * x, [0.0]]).astype(np.float32))
        for edge in (3.5, 7.0):  # of the scale rule, on either side of it
            for t in (np.nextafter(np.float32(edge * 2.0 ** k), np.float32(0)), np.float32(edge * 2.0 ** k),
                      np.nextafter(np.float32(edge * 2.0 ** k), np.float32(np.inf))):
                groups.append(np.concatenate([[-t], np.minimum(x, t), [-0.0]]).astype(np.float32))
    return np.array(groups)


@pytest.mark.parametrize("append", [False, True])
def test_numbers_beside_borders(append):
    x = rows()
    assert np.isfinite(x).all() and (np.abs(x[x != 0]) < 2.0 ** -126).any()
    C = -(-len(x) // 2)
    x = np.concatenate([x, np.zeros((2 * C - len(x), 32), np.float32)]).reshape(1, 1, C, 64)
    K = torch.as_tensor(x).cuda()
    shape = rk.make_shape(1, 1, 1, 64, "f32", C, 1)
    cache, lens = filled(shape, 0), i32([0 if append else C])
    if append:
        rk.reskv_append_kv_quant(shape, K, K, cache, i32([0]), lens)
    else:
        rk.reskv_pack_quant(shape, K, K, i32([0]), lens, cache)
    want = ref.pack(host(K), host(K), [[C]])
    assert (cache.cpu().numpy().reshape(want.shape) == want).all() and lens.tolist() == [C]
    ko, vo = torch.empty_like(K), torch.empty_like(K)
    rk.reskv_unpack_quant(shape, cache, i32([0]), lens, ko, vo)
    value = ref.quantize(host(K))[0]
    assert (host(ko) == value).all() and (host(vo) == value).all()
