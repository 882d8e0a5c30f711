"""Decode over 4-bit caches whose heads are split over several blocks and joined by a second launch, as a serving loop
runs it: rotation, appended tokens, lengths that the join advances, full caches, borders of the parts, replays, NaN and
empty records. Then, split or not, corrupt lengths and the gate's edge settings."""

import ctypes

import numpy as np
import pytest
import torch

from oracle import reskv_oracle as orc
from paper_2607_29591_amd import reskv as rk
from tests import quant_ref as ref
from tests.test_quant_decode_gpu import DT, Case, dev, host, i32

pytestmark = pytest.mark.gpu
C = 3000     # six parts of eight cache blocks for up to 42 pairs
PART = 512


def parts(shape):
    return rk.lib().reskv_internal_quant_parts(ctypes.byref(shape))


@pytest.mark.parametrize("dtype,d,G", [("bf16", 128, 4), ("bf16", 64, 7), ("f32", 128, 2), ("f32", 64, 16)])
@pytest.mark.parametrize("layout,part", [("half", 1.0), ("interleaved", 0.5)])
def test_step_is_the_calls_in_a_row(dtype, d, G, layout, part):
    """Rotation, append and decode in one call: the same bits as the three calls, and the oracle's output. Heads: one
    full, one that fills its last slot, appends on the first slot of a part and of a cache block, residual slots up to
    a part's border and past one, a head of one slot."""
    B, H = 4, 2
    r = np.array([[5, 700], [0, 512], [512, 511], [0, 1030]])
    n = np.array([[C - 5, C - 701], [1024, 512], [64, 1], [1, 506]])
    c = Case(7, dtype, d, B, H, G, C, 1100, r, n)
    assert parts(c.shape) == 6
    plan = rk.make_rope(int(d * part), layout=layout, scaling="llama3", theta=500000.0, factor=8.0, original_len=8192.0)
    pos = i32([3, 70000, 131071, 0])
    fused_cache, fused_len = c.cache.clone(), c.main_len.clone()
    fused = c.decode({}, append=True, rope=plan, positions=pos, cache=fused_cache, main_len=fused_len)
    q = torch.empty_like(c.q)
    rk.reskv_rope(c.shape, plan, pos.reshape(B, 1), q=c.q.reshape(B, G * H, 1, d), q_out=q.reshape(B, G * H, 1, d))
    rk.reskv_append_kv_quant(c.shape, c.k_new, c.v_new, c.cache, c.res_len, c.main_len, rope=plan, positions=pos)
    alone = c.decode({}, q=q)
    after = np.minimum(n + 1, C - r)
    assert (fused_len.cpu().numpy().reshape(B, H) == after).all() and torch.equal(c.main_len, fused_len)
    assert torch.equal(c.cache, fused_cache)
    for a, b in zip(fused, alone):
        assert torch.equal(a, b)
    K, V = (torch.zeros(B, H, C, d, dtype=DT[dtype], device="cuda") for _ in range(2))
    rk.reskv_unpack_quant(c.shape, c.cache, c.res_len, c.main_len, K, V)
    c.check(fused, {}, q=host(q), K=host(K), V=host(V), n=after)


@pytest.mark.parametrize("r,n", [(0, 1), (0, 512), (0, 513), (512, 1), (512, 512), (513, 511), (1, 1023), (1100, 1),
                                 (700, 2300), (1024, 1976), (2999, 1)])
def test_lengths_at_the_borders_of_the_parts(r, n):
    """Slots past the live ones hold 0xFF; the workspace too, so that a record that was not written shows."""
    c = Case(r + n, "bf16", 128, 1, 1, 4, C, max(r, 1), [[r]], [[n]])
    assert parts(c.shape) == 6
    c.check(c.decode({}), {})


def test_a_workspace_keeps_nothing():
    """Long lengths, then short ones, in one workspace: what a fresh one gives."""
    c = Case(18, "bf16", 128, 1, 2, 4, C, 700, [[600, 0]], [[2400, 3000]])
    ws = torch.full((rk.reskv_decode_quant_workspace_size(c.shape),), 0xFF, dtype=torch.uint8, device="cuda")
    outs = []
    for res, main in ([600, 0], [2400, 3000]), ([3, 0], [1, 5]):
        rl, ml = i32(res), i32(main)
        out = torch.empty(1, 8, 128, device="cuda")
        rk.reskv_decode_attn_quant(c.shape, rk.make_gate(), c.q, c.cache, c.logc_dev, rl, ml, out, ws)
        outs.append(out)
        fresh = torch.empty_like(out)
        rk.reskv_decode_attn_quant(c.shape, rk.make_gate(), c.q, c.cache, c.logc_dev, rl, ml, fresh,
                                   torch.full_like(ws, 0xFF))
        assert torch.equal(out, fresh)
    assert not torch.equal(*outs)


def test_graph_replays_match_eager_steps():
    """A captured step replayed with new inputs and eager steps between: over a part's border, into a full cache, and
    from no main slot."""
    B, H, G, d = 2, 2, 4, 128
    c = Case(17, "bf16", d, B, H, G, C, 600, [[10, 512], [0, 600]], [[500, 1], [2998, 1]])
    assert parts(c.shape) == 6
    c.n = np.array([[500, 0], [2998, 0]])
    c.main_len = i32(c.n)
    plan, pos = rk.make_rope(d), i32([10, 20])
    caches, lens = [c.cache.clone(), c.cache.clone()], [c.main_len.clone(), c.main_len.clone()]
    outs = [torch.zeros(B, G * H, d, device="cuda") for _ in range(2)]
    wss = [torch.zeros(rk.reskv_decode_quant_workspace_size(c.shape), dtype=torch.uint8, device="cuda")
           for _ in range(2)]

    def call(i):
        rk.reskv_decode_attn_quant(c.shape, rk.make_gate(), c.q, caches[i], c.logc_dev, c.res_len, lens[i], outs[i],
                                   wss[i], rope=plan, positions=pos, k_new=c.k_new, v_new=c.v_new)

    call(0)
    caches[0].copy_(c.cache)
    lens[0].copy_(c.main_len)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(1)
    for step in range(6):
        c.q.copy_(dev(c.rng.normal(size=c.q.shape), "bf16"))
        c.k_new.copy_(dev(c.rng.normal(size=c.k_new.shape), "bf16"))
        c.v_new.copy_(dev(c.rng.normal(size=c.v_new.shape), "bf16"))
        pos.add_(1)
        torch.cuda.synchronize()
        g.replay()
        call(0)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.equal(lens[0], lens[1]) and torch.equal(caches[0], caches[1])
        n = np.minimum(c.n + step + 1, C - c.r)
        assert (lens[1].cpu().numpy().reshape(B, H) == n).all()
        K, V = (torch.zeros(B, H, C, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        rk.reskv_unpack_quant(c.shape, caches[1], c.res_len, lens[1], K, V)
        turned = torch.empty(B, G * H, 1, d, dtype=torch.bfloat16, device="cuda")
        rk.reskv_rope(c.shape, plan, pos.reshape(B, 1), q=c.q.reshape(B, G * H, 1, d), q_out=turned)
        want = orc.decode(host(turned)[:, :, 0], host(K), host(V), c.logc.astype(np.float32), c.r, n, 0.25, 12.0, 0.0, 1.0)
        for b in range(B):
            for h in range(G * H):
                kv = h // G
                live = np.concatenate([np.isfinite(c.logc[b, kv, :c.r[b, kv]]), np.ones(n[b, kv], bool)])
                Kl, Vl = (host(x)[b, kv, :c.r[b, kv] + n[b, kv]][live] for x in (K, V))
                tol = ref.decode_atol(host(turned)[b, h, 0], Kl, Vl, want[3][b, h], want[1][b, h], 12.0, 0.0)
                assert np.abs(host(outs[1])[b, h] - want[0][b, h]).max() <= tol, (step, b, h)


def test_empty_entries_and_dead_slots_hold_anything():
    c = Case(11, "bf16", 128, 1, 2, 4, C, 900, [[900, 40]], [[500, 2000]], fill=0, empty=0.5)
    assert parts(c.shape) == 6
    a = c.decode({})
    pk, pv, sk, sv = ref.places(128, C)
    bad = c.cache.cpu().numpy().reshape(2, -1).copy()
    for h in range(2):
        dead = [j for j in range(c.r[0, h]) if not np.isfinite(c.logc[0, h, j])]
        dead += list(range(c.r[0, h] + c.n[0, h], C))
        assert len(dead) > 900
        for j in dead:
            bad[h, sk[j]] = bad[h, sv[j]] = 255
            bad[h, pk[j]] = bad[h, pv[j]] = 0x77
    c.cache.copy_(torch.as_tensor(bad.reshape(-1)))
    for x, y in zip(a, c.decode({})):
        assert torch.equal(x, y)


def test_no_live_slot_and_no_main_slot():
    """A head without live slots gives 0; one with entries only their own softmax (p_max is taken as 1)."""
    H, G, d = 3, 4, 128
    c = Case(12, "bf16", d, 1, H, G, C, 700, [[0, 700, 700]], [[20, 20, 20]], empty=0.0)
    assert parts(c.shape) == 6
    c.main_len.zero_()
    c.logc_dev[0, 2] = -float("inf")
    out, lse_main, lse_res, gate = c.decode({})
    assert not out[0, :G].any() and not out[0, 2 * G:].any()
    assert (lse_main == -float("inf")).all()
    assert (lse_res[0, :G] == -float("inf")).all() and (lse_res[0, 2 * G:] == -float("inf")).all()
    for h in range(G, 2 * G):
        q, K, V, lc = host(c.q)[0, h], c.K[0, 1, :700], c.V[0, 1, :700], c.logc[0, 1, :700].astype(np.float32)
        a = K @ q / np.sqrt(d) + lc
        w = np.exp(a - a.max())
        assert np.abs(host(out)[0, h] - w @ V / w.sum()).max() <= ref.decode_atol(q, K, V, 1.0, 0.0, 12.0, 0.0)


@pytest.mark.parametrize("first,count", [(1600, 1), (1536, 512), (0, 3000)])
def test_nan_keys_reach_the_output(first, count):
    """One NaN key, a whole part of them (its record has no maximum), every key."""
    c = Case(13, "bf16", 64, 1, 2, 2, C, 10, [[0, 0]], [[3000, 3000]])
    assert parts(c.shape) == 6
    before = c.decode({})[0]
    kc, vc = dev(c.K, "bf16"), dev(c.V, "bf16")
    kc[0, 0, first:first + count] = float("nan")
    rk.reskv_pack_quant(c.shape, kc, vc, c.res_len, c.main_len, c.cache)
    out = c.decode({})[0]
    assert torch.isnan(out[0, :2]).all() and torch.isfinite(out[0, 2:]).all()
    assert torch.equal(out[0, 2:], before[0, 2:])  # 4-bit values code to themselves


def test_one_huge_key_of_a_late_part_dominates():
    c = Case(14, "bf16", 64, 1, 2, 2, C, 600, [[600, 0]], [[2400, 3000]])
    assert parts(c.shape) == 6
    kc, vc = torch.zeros(1, 2, C, 64, dtype=torch.bfloat16, device="cuda"), dev(c.V, "bf16")
    kc[0, :, 2100] = 3.0e38
    rk.reskv_pack_quant(c.shape, kc, vc, c.res_len, c.main_len, c.cache)
    c.q.abs_().mul_(1e-30)
    out = host(c.decode({})[0])
    want = c.V[0, :, 2100].repeat(2, 0)
    # its probability p in [1, 2) 2^k enters as two bf16 parts: the first is off by r <= 2^-8 2^k, half of a step of
    # 2^-7 2^k; r lies below 2^-8 2^k or is it, so the second is off by at most half of a step of 2^-16 2^k: 2^-17 of
    # p. The denominator, its reciprocal, the products of the weights and the sums that only add zeros round eight
    # times, 2^-24 each.
    assert (np.abs(out[0] - want) <= (2.0 ** -17 + 8 * 2.0 ** -24) * np.abs(want)).all()


# ------------------------------------------------------- split or not

BIG = 2 ** 31 - 1
CORRUPT = ([-5, BIG, 3, 8], [BIG, 50, -1, BIG])


def guarded(count, dtype=torch.uint8, fill=0):
    """A tensor of `count` elements with 4096 others on both sides, and whether those are as they were."""
    buf = torch.full((count + 8192,), 77, dtype=dtype, device="cuda")
    buf[4096:4096 + count] = fill
    return buf[4096:4096 + count], lambda: bool((buf[:4096] == 77).all() and (buf[4096 + count:] == 77).all())


def clamped(res, main, Ccap, Rcap):
    r = np.clip(res, 0, min(Rcap, Ccap))
    return r, np.clip(main, 0, Ccap - r)


@pytest.mark.parametrize("n_new", [1, 5, 20, 150])
def test_append_with_corrupt_lengths_stays_inside(n_new):
    """What the lengths within the capacities give; nothing outside of the cache or of the lengths is written."""
    Ccap, d, H = 100, 64, 4
    rng = np.random.default_rng(n_new)
    shape = rk.make_shape(1, H, H, d, "bf16", Ccap, 8)
    r, n = clamped(*CORRUPT, Ccap, 8)
    k, v = (dev(rng.normal(size=(1, H, n_new, d)), "bf16") for _ in range(2))
    cache, whole = guarded(rk.reskv_quant_cache_size(shape))
    lens, lens_whole = guarded(H, torch.int32)
    lens.copy_(i32(CORRUPT[1]))
    rk.reskv_append_kv_quant(shape, k, v, cache, i32(CORRUPT[0]), lens)
    want, want_len = torch.zeros_like(cache), i32(n)
    rk.reskv_append_kv_quant(shape, k, v, want, i32(r), want_len)
    assert torch.equal(cache, want) and whole() and lens_whole()
    took = want_len.cpu().numpy() > n
    assert (lens.cpu().numpy() == np.where(took, want_len.cpu().numpy(), CORRUPT[1])).all()
    assert took.tolist() == [False, True, True, False]


def test_unpack_with_corrupt_lengths_stays_inside():
    Ccap, d, H, rows = 100, 64, 4, 130
    rng = np.random.default_rng(1)
    shape = rk.make_shape(1, H, H, d, "bf16", Ccap, 8)
    x = dev(rng.normal(size=(1, H, Ccap, d)), "bf16")
    cache = torch.zeros(rk.reskv_quant_cache_size(shape), dtype=torch.uint8, device="cuda")
    rk.reskv_pack_quant(shape, x, x, i32([0] * H), i32([Ccap] * H), cache)
    r, n = clamped(*CORRUPT, Ccap, 8)
    k, k_whole = guarded(H * rows * d, torch.bfloat16, 5.0)
    v, v_whole = guarded(H * rows * d, torch.bfloat16, 5.0)
    rk.reskv_unpack_quant(shape, cache, i32(CORRUPT[0]), i32(CORRUPT[1]), k.view(1, H, rows, d), v.view(1, H, rows, d))
    want = np.full((1, H, rows, d), 5.0)
    for h in range(H):
        want[0, h, :r[h] + n[h]] = ref.quantize(host(x))[0][0, h, :r[h] + n[h]]
    assert k_whole() and v_whole()
    assert (host(k).reshape(want.shape) == want).all() and (host(v).reshape(want.shape) == want).all()


@pytest.mark.parametrize("Ccap,Rcap,split", [(100, 8, 1), (100, 300, 1), (C, 8, 6), (C, 4000, 6)])
@pytest.mark.parametrize("append", [False, True])
def test_decode_with_corrupt_lengths_stays_inside(Ccap, Rcap, split, append):
    """The bits that the lengths within the capacities give, also where more entries are named than there are slots."""
    H, G, d = 4, 2, 64
    res, main = ([-5, BIG, 3, 8] if Rcap == 8 else [BIG, Ccap + 50, 3, -1]), CORRUPT[1]
    r, n = clamped(res, main, Ccap, Rcap)
    c = Case(Ccap + Rcap, "bf16", d, 1, H, G, Ccap, Rcap, [np.minimum(r, Ccap - 1)], [np.maximum(n, 1)])
    assert parts(c.shape) == split
    cache, whole = guarded(c.cache.numel())
    cache.copy_(c.cache)
    lens, lens_whole = guarded(H, torch.int32)
    out, out_whole = guarded(H * G * d, torch.float32)
    ws, ws_whole = guarded(rk.reskv_decode_quant_workspace_size(c.shape), fill=0xFF)
    new = dict(k_new=c.k_new, v_new=c.v_new) if append else {}
    lens.copy_(i32(main))
    rk.reskv_decode_attn_quant(c.shape, rk.make_gate(), c.q, cache, c.logc_dev, i32(res), lens, out, ws, **new)
    want, want_len = torch.empty_like(out), i32(n)
    rk.reskv_decode_attn_quant(c.shape, rk.make_gate(), c.q, c.cache, c.logc_dev, i32(r), want_len, want,
                               torch.full_like(ws, 0xFF), **new)
    assert whole() and lens_whole() and out_whole() and ws_whole()
    assert torch.equal(out, want) and torch.equal(cache, c.cache) and torch.isfinite(out).all()
    room = np.asarray(r) + n < Ccap
    assert (want_len.cpu().numpy() == (n + (room & append))).all()
    assert (lens.cpu().numpy() == np.where(room & append, n + 1, main)).all()


# no count weighting, a constant gate of 1/2, the gate pinned at 1, a threshold far below every p_max (the gate
# underflows: entries off) and far above it (gate 1)
GATE_EDGES = [dict(beta=0.0), dict(alpha=0.0), dict(alpha=0.0, g_min=1.0, beta=0.0), dict(tau_scalar=-50.0),
              dict(tau_scalar=50.0), dict(g_min=1.0), dict(tau_scalar=0.9, alpha=3.0, g_min=0.2, beta=0.5)]


@pytest.mark.parametrize("Ccap,split", [(400, 1), (2100, 5)])
@pytest.mark.parametrize("gate", GATE_EDGES)
def test_gate_edges(Ccap, split, gate):
    c = Case(19, "bf16", 128, 2, 2, 4, Ccap, 300)
    assert parts(c.shape) == split
    c.check(c.decode(gate), gate)
