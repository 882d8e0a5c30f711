"""Every check that the binding of the rotation and the 4-bit caches makes of a tensor, one wrong property at a time:
all tensors lie on the GPU, so that the check meant is the one that refuses, and each call is made once with nothing
wrong."""

import pytest
import torch

from paper_2607_29591_amd import reskv as rk

pytestmark = pytest.mark.gpu
B, Hq, H, d, C, Rcap, n = 2, 8, 2, 128, 70, 8, 3
BF, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


def shape():
    return rk.make_shape(B, Hq, H, d, "bf16", C, Rcap)


def zeros(dtype, *size):
    return torch.zeros(*size, dtype=dtype, device="cuda")


def arguments(call):
    """Tensors of a call that is taken."""
    lens = dict(cache=zeros(U8, rk.reskv_quant_cache_size(shape())), res_len=zeros(I32, B * H), main_len=zeros(I32, B * H))
    return {
        "rope": lambda: dict(positions=zeros(I32, B, n), q=zeros(BF, B, Hq, n, d), q_out=zeros(BF, B, Hq, n, d),
                             k=zeros(BF, B, H, n, d), k_out=zeros(BF, B, H, n, d), n_tok=zeros(I32, B)),
        "pack": lambda: dict(kc=zeros(BF, B, H, C, d), vc=zeros(BF, B, H, C, d), **lens),
        "unpack": lambda: dict(kc=zeros(BF, B, H, n, d), vc=zeros(BF, B, H, n, d), first_slot=zeros(I32, B * H), **lens),
        "append": lambda: dict(k_new=zeros(BF, B, H, n, d), v_new=zeros(BF, B, H, n, d), positions=zeros(I32, B, n),
                               n_tok=zeros(I32, B), **lens),
        "decode": lambda: dict(q=zeros(BF, B, Hq, d), logc=zeros(F32, B, H, Rcap), out=zeros(F32, B, Hq, d),
                               workspace=zeros(U8, rk.reskv_decode_quant_workspace_size(shape())),
                               positions=zeros(I32, B), dbg_lse_main=zeros(F32, B * Hq), dbg_lse_res=zeros(F32, B * Hq),
                               dbg_gate=zeros(F32, B * Hq), k_new=zeros(BF, B, H, d), v_new=zeros(BF, B, H, d),
                               tau=zeros(F32, B, Hq), **lens)}[call]()


def issue(call, a, plan):
    a, s = dict(a), shape()
    if call == "rope":
        rk.reskv_rope(s, plan, **a)
    elif call == "pack":
        rk.reskv_pack_quant(s, **a)
    elif call == "unpack":
        rk.reskv_unpack_quant(s, **a)
    elif call == "append":
        rk.reskv_append_kv_quant(s, rope=plan, **a)
    else:
        rk.reskv_decode_attn_quant(s, rk.make_gate(tau=a.pop("tau")), rope=plan, **a)
    torch.cuda.synchronize()


def columns(t):
    """The same shape with every other element of a wider tensor."""
    return torch.zeros(*t.shape[:-1], 2 * t.shape[-1], dtype=t.dtype, device=t.device)[..., ::2]


WRONG = {"type": (lambda t: t.to(torch.float64), "must be torch"),
         "size": (lambda t: t[..., :-1].contiguous(), r"must (be \[|have)"),
         "place": (lambda t: t.cpu(), "must be on the current GPU"),
         "order": (columns, r"must be (contiguous|\[.* adjoining)")}


@pytest.mark.parametrize("call", ["rope", "pack", "unpack", "append", "decode"])
def test_every_wrong_tensor_is_named(call):
    plan, good = rk.make_rope(64), arguments(call)
    issue(call, good, plan)
    for name in set(good) - {"workspace"}:
        for wrong, (change, match) in WRONG.items():
            match = f"{name} {match}"
            if (call, name, wrong) == ("rope", "positions", "size"):  # they say how many rows there are
                match = r"q must be \[2, 8, 2, 128\]"
            if (name, wrong) == ("tau", "order"):  # refused where the gate is made
                match = "must be contiguous"
            with pytest.raises(ValueError, match=match):
                issue(call, dict(good, **{name: change(good[name])}), plan)


@pytest.mark.parametrize("wrong", ["small", "place", "order"])
def test_wrong_workspaces(wrong):
    plan, a = rk.make_rope(64), arguments("decode")
    ws = a["workspace"]
    a["workspace"] = {"small": ws[:16], "place": ws.cpu(), "order": columns(ws)}[wrong]
    with pytest.raises(rk.ReskvError if wrong == "small" else ValueError,
                       match={"small": "workspace", "place": "current GPU", "order": "contiguous"}[wrong]):
        issue("decode", a, plan)
