"""Rotations between slices of one buffer on the GPU, against the same rows rotated apart from each other."""

import numpy as np
import pytest
import torch

from paper_2607_29591_amd import reskv as rk

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def positions(B, n):
    return (torch.arange(B * n, dtype=torch.int32, device="cuda") * 37 % 5000).reshape(B, n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,n,d", [(1, 1, 128), (2, 33, 64), (3, 300, 128)])
def test_from_columns_into_columns_of_one_buffer(dtype, B, n, d):
    """Queries from the first columns of a buffer's rows into later ones, between the keys and values that lie there,
    and keys into columns of every other head."""
    rng = np.random.default_rng(n)
    Hq, H = 4, 2
    buf = torch.as_tensor(rng.normal(size=(B, n, 16, d)), dtype=torch.float32).to(DT[dtype]).cuda()
    want, x = buf.clone(), buf.transpose(1, 2)
    q, k, pos = x[:, :Hq], x[:, Hq:Hq + H], positions(B, n)
    shape, rope = rk.make_shape(B, Hq, H, d, dtype, 1, 1), rk.make_rope(32)
    apart_q, apart_k = torch.empty_like(q.contiguous()), torch.empty_like(k.contiguous())
    rk.reskv_rope(shape, rope, pos, q=q.contiguous(), q_out=apart_q, k=k.contiguous(), k_out=apart_k)
    want.transpose(1, 2)[:, 6:10] = apart_q
    want.transpose(1, 2)[:, 11:15:2] = apart_k
    rk.reskv_rope(shape, rope, pos, q=q, q_out=x[:, 6:10], k=k, k_out=x[:, 11:15:2])
    assert torch.equal(buf, want)
