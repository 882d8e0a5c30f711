"""Decode over 4-bit caches against the oracle's decode of the values the codes stand for, and the whole run of the
rotation, the packing, the appends and the decode steps."""

import numpy as np
import pytest
import torch

from oracle import reskv_oracle as orc
from paper_2607_29591_amd import reskv as rk
from tests import quant_ref as ref
from tests.helpers import gate_atol, random_cache

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def host(t):
    return t.detach().double().cpu().numpy()


def dev(x, dtype):
    return torch.as_tensor(np.asarray(x), dtype=torch.float32).to(DT[dtype]).cuda().contiguous()


def i32(x):
    return torch.as_tensor(np.asarray(x, np.int32).reshape(-1)).cuda()


class Case:
    """A packed cache, queries and a token, on both sides."""

    def __init__(self, seed, dtype, d, B, H, G, C, Rcap, res=None, main=None, fill=0xFF, empty=0.1, scale=1.0):
        rng = self.rng = np.random.default_rng(seed)
        self.dtype, self.d, self.B, self.H, self.G, self.C = dtype, d, B, H, G, C
        self.r = np.asarray(res) if res is not None else rng.integers(0, min(Rcap, C - 1) + 1, size=(B, H))
        self.n = np.asarray(main) if main is not None else \
            np.array([[int(rng.integers(1, C - x + 1)) for x in row] for row in self.r])
        kc, vc, self.logc = random_cache(rng, B, H, C, Rcap, d, dtype, self.r, np.maximum(self.n, 1), empty, scale)
        self.shape = rk.make_shape(B, G * H, H, d, dtype, C, Rcap)
        self.cache = torch.full((rk.reskv_quant_cache_size(self.shape),), fill, dtype=torch.uint8, device="cuda")
        self.res_len, self.main_len = i32(self.r), i32(self.n)
        rk.reskv_pack_quant(self.shape, dev(kc, dtype), dev(vc, dtype), self.res_len, self.main_len, self.cache)
        self.K, self.V = ref.quantize(kc)[0], ref.quantize(vc)[0]
        self.q = dev(rng.normal(size=(B, G * H, d)) * 1.3, dtype)
        self.k_new, self.v_new = dev(rng.normal(size=(B, H, d)), dtype), dev(rng.normal(size=(B, H, d)), dtype)
        self.logc_dev = torch.as_tensor(self.logc.astype(np.float32)).cuda()

    def decode(self, gate_kw, tau=None, append=False, rope=None, positions=None, q=None, cache=None, main_len=None):
        B, Hq = self.B, self.G * self.H
        out = torch.full((B, Hq, self.d), float("nan"), device="cuda")
        stats = [torch.full((B * Hq,), float("nan"), device="cuda") for _ in range(3)]
        ws = torch.full((rk.reskv_decode_quant_workspace_size(self.shape),), 0xFF, dtype=torch.uint8, device="cuda")
        gate = rk.make_gate(tau=tau, **gate_kw)
        new = dict(k_new=self.k_new, v_new=self.v_new) if append else {}
        rk.reskv_decode_attn_quant(self.shape, gate, self.q if q is None else q,
                                   self.cache if cache is None else cache, self.logc_dev, self.res_len,
                                   self.main_len if main_len is None else main_len, out, ws, rope=rope,
                                   positions=positions, dbg_lse_main=stats[0], dbg_lse_res=stats[1],
                                   dbg_gate=stats[2], **new)
        torch.cuda.synchronize()
        return [out] + [s.reshape(B, Hq) for s in stats]

    def check(self, got, gate_kw, tau=None, q=None, K=None, V=None, n=None):
        q, K, V, n = (host(self.q) if q is None else q, self.K if K is None else K, self.V if V is None else V,
                      self.n if n is None else n)
        gate_kw = dict(dict(tau_scalar=0.25, alpha=12.0, g_min=0.0, beta=1.0), **gate_kw)
        logc = self.logc.astype(np.float32).astype(np.float64)
        want = orc.decode(q, K, V, logc, self.r, n, gate_kw["tau_scalar"] if tau is None else host(tau),
                          gate_kw["alpha"], gate_kw["g_min"], gate_kw["beta"])
        for b in range(self.B):
            for h in range(self.G * self.H):
                kv = h // self.G
                r, m = int(self.r[b, kv]), int(n[b, kv])
                live = np.concatenate([np.isfinite(logc[b, kv, :r]), np.ones(m, bool)])
                Kl, Vl = K[b, kv, :r + m][live], V[b, kv, :r + m][live]
                g, lse = want[3][b, h], want[1][b, h]
                mag = float((np.abs(Kl) @ np.abs(q[b, h])).max()) / np.sqrt(self.d)
                lse_tol = (3 * self.d + 8) * 2.0 ** -24 * mag + 2.0 ** -20 + 2.0 ** -22 * abs(lse) + m * 2.0 ** -26
                assert abs(host(got[1])[b, h] - lse) <= lse_tol, (b, h, "lse_main")
                if np.isfinite(want[2][b, h]):
                    assert abs(host(got[2])[b, h] - want[2][b, h]) <= lse_tol + 2.0 ** -22 * abs(want[2][b, h])
                else:
                    assert host(got[2])[b, h] == -np.inf
                tol_g = 3 * gate_atol(q[b, h], K[b, kv, r:r + m], g, lse, gate_kw["alpha"])
                assert abs(host(got[3])[b, h] - g) <= tol_g, (b, h, "gate")
                tol = ref.decode_atol(q[b, h], Kl, Vl, g, lse, gate_kw["alpha"], gate_kw["g_min"])
                off = np.abs(host(got[0])[b, h] - want[0][b, h]).max()
                assert off <= tol, (b, h, off, tol)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("G", [1, 2, 3, 4, 7, 8, 16])
def test_group_sizes(dtype, d, G):
    c = Case(G, dtype, d, 2, 2, G, 333, 70)
    c.check(c.decode({}), {})


@pytest.mark.parametrize("r,n", [(0, 1), (0, 63), (0, 64), (0, 65), (1, 1), (1, 63), (63, 1), (64, 64), (64, 1),
                                 (65, 127), (100, 412), (0, 513), (130, 1100), (1000, 25), (255, 257)])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
def test_lengths(dtype, d, r, n):
    """Slots past the live ones hold 0xFF: codes of -6 and scales that stand for NaN."""
    c = Case(r + n, dtype, d, 1, 1, 4, r + n + 3, max(r, 1), [[r]], [[n]])
    c.check(c.decode({}), {})


@pytest.mark.parametrize("seed", range(24))
def test_random_shapes(seed):
    rng = np.random.default_rng(100 + seed)
    dtype, d = [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)][seed % 4]
    G, H, B = int(rng.choice([1, 2, 4, 5, 7, 8, 12, 16])), int(rng.choice([1, 2, 4])), int(rng.integers(1, 5))
    C = int(rng.integers(8, 2600))
    c = Case(seed, dtype, d, B, H, G, C, int(rng.integers(1, 600)))
    gate = dict(tau_scalar=float(rng.uniform(0.05, 0.6)), alpha=float(rng.choice([4.0, 12.0])),
                g_min=float(rng.choice([0.0, 0.2])), beta=float(rng.choice([0.5, 1.0])))
    tau = torch.as_tensor(rng.normal(0.3, 0.2, size=(B, G * H)), dtype=torch.float32).cuda() if seed % 3 == 0 else None
    c.check(c.decode(gate, tau=tau), gate, tau=tau)


@pytest.mark.parametrize("dtype,d,G", [("bf16", 128, 4), ("bf16", 64, 7), ("f32", 128, 2), ("f32", 64, 16)])
@pytest.mark.parametrize("layout,part", [("half", 1.0), ("interleaved", 0.5)])
def test_fused_step_is_the_calls_in_a_row(dtype, d, G, layout, part):
    """Rotation, append and decode in one call: the same bits as the three calls; lengths and cache too. One head is
    full (nothing is appended), one fills its last slot, one starts a block."""
    B, H, C = 3, 2, 320
    r = np.array([[5, 30], [0, 64], [17, 0]])
    n = np.array([[60, C - 30], [C - 1, 128], [111, 1]])
    c = Case(7, dtype, d, B, H, G, C, 70, r, n)
    plan = rk.make_rope(int(d * part), layout=layout, scaling="llama3", theta=500000.0, factor=8.0, original_len=8192.0)
    pos = i32([3, 70000, 131071])
    fused_cache, fused_len = c.cache.clone(), c.main_len.clone()
    fused = c.decode({}, append=True, rope=plan, positions=pos, cache=fused_cache, main_len=fused_len)
    q = torch.empty_like(c.q)
    rk.reskv_rope(c.shape, plan, pos.reshape(B, 1), q=c.q.reshape(B, G * H, 1, d), q_out=q.reshape(B, G * H, 1, d))
    rk.reskv_append_kv_quant(c.shape, c.k_new, c.v_new, c.cache, c.res_len, c.main_len, rope=plan, positions=pos)
    alone = c.decode({}, q=q)
    assert torch.equal(c.cache, fused_cache) and torch.equal(c.main_len, fused_len)
    assert c.main_len.reshape(B, H).tolist() == np.minimum(n + 1, C - r).tolist()
    for a, b in zip(fused, alone):
        assert torch.equal(a, b)
    K, V = (torch.zeros(B, H, C, d, dtype=DT[dtype], device="cuda") for _ in range(2))
    rk.reskv_unpack_quant(c.shape, c.cache, c.res_len, c.main_len, K, V)
    c.check(fused, {}, q=host(q), K=host(K), V=host(V), n=np.minimum(n + 1, C - r))


def test_empty_entries_and_dead_slots_hold_anything():
    """Empty entries and slots past the end may hold NaN and infinities: outputs keep their bits."""
    c = Case(11, "bf16", 128, 1, 2, 4, 200, 90, [[90, 40]], [[50, 0]], fill=0, empty=0.5)
    n = np.array([[50, 30]])
    c.n, c.main_len = n, i32(n)
    a = c.decode({})
    pk, pv, sk, sv = ref.places(128, 200)
    bad = c.cache.cpu().numpy().reshape(2, -1).copy()
    for h in range(2):
        dead = [j for j in range(c.r[0, h]) if not np.isfinite(c.logc[0, h, j])]
        dead += list(range(c.r[0, h] + n[0, h], 200))
        assert len(dead) > 60
        for j in dead:
            bad[h, sk[j]] = bad[h, sv[j]] = 255
            bad[h, pk[j]] = bad[h, pv[j]] = 0x77
    c.cache.copy_(torch.as_tensor(bad.reshape(-1)))
    for x, y in zip(a, c.decode({})):
        assert torch.equal(x, y)


def test_no_live_slot_and_no_main_slot():
    """A head without live slots gives 0; one with entries only gives their own softmax (p_max is taken as 1)."""
    B, H, G, d, C = 1, 3, 4, 128, 80
    c = Case(12, "bf16", d, B, H, G, C, 40, [[0, 40, 40]], [[20, 20, 20]], empty=0.0)
    c.main_len.zero_()
    c.logc_dev[0, 2] = -float("inf")
    out, lse_main, lse_res, gate = c.decode({})
    assert not out[0, :G].any() and not out[0, 2 * G:].any()
    assert (lse_main == -float("inf")).all() and (lse_res[0, 2 * G:] == -float("inf")).all()
    for h in range(G, 2 * G):
        q, K, V, lc = host(c.q)[0, h], c.K[0, 1, :40], c.V[0, 1, :40], c.logc[0, 1, :40].astype(np.float32)
        a = K @ q / np.sqrt(d) + lc
        w = np.exp(a - a.max())
        assert np.abs(host(out)[0, h] - w @ V / w.sum()).max() <= ref.decode_atol(q, K, V, 1.0, 0.0, 12.0, 0.0)


def test_nan_and_huge_keys_reach_the_output():
    c = Case(13, "bf16", 64, 1, 2, 2, 130, 10)
    kc = torch.zeros(1, 2, 130, 64, dtype=torch.bfloat16, device="cuda")
    kc[0, 0, int(c.r[0, 0])] = float("nan")
    kc[0, 1, int(c.r[0, 1])] = 3.0e38  # one key dominates: its value comes out
    c.q.abs_()
    vc = dev(c.rng.normal(size=(1, 2, 130, 64)), "bf16")
    rk.reskv_pack_quant(c.shape, kc, vc, c.res_len, c.main_len, c.cache)
    out = c.decode({})[0]
    assert torch.isnan(out[0, :2]).all()
    c.main_len.clamp_(max=1)  # and where nothing but that key is left
    c.logc_dev.fill_(-float("inf"))
    assert torch.isnan(c.decode({})[0][0, :2]).all()
    c.main_len.copy_(i32(c.n))
    c.q.mul_(1e-30)
    out = c.decode({})[0]
    want = torch.as_tensor(ref.quantize(host(vc))[0][0, 1, int(c.r[0, 1])]).cuda()
    assert ((out[0, 2:].double() - want).abs() <= 2.0 ** -17 * want.abs().max()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_and_many(dtype):
    """One long cache with many entries, and 260 pairs."""
    c = Case(14, dtype, 128, 1, 1, 4, 9000, 4096, [[2000]], [[6999]])
    c.check(c.decode({}), {})
    c = Case(15, dtype, 64, 65, 4, 2, 150, 40)
    c.check(c.decode({}), {})


def test_offsets_past_32_bits():
    """A cache of more than 2^32 bytes: the last heads decode as they do in a small cache of their own."""
    d, G, H, C = 128, 2, 64, 8192
    B = -(-(2 ** 32 + 2 ** 28) // (H * C // 64 * 68 * d))
    shape = rk.make_shape(B, G * H, H, d, "bf16", C, 1)
    small = Case(16, "bf16", d, 1, H, G, C, 1, np.zeros((1, H), int), np.full((1, H), 200))
    cache = torch.empty(rk.reskv_quant_cache_size(shape), dtype=torch.uint8, device="cuda")
    assert cache.numel() > 2 ** 32
    cache[-small.cache.numel():] = small.cache
    main = np.zeros((B, H), int)
    main[-1] = 200
    rl, ml = i32(np.zeros((B, H))), i32(main)
    q = torch.zeros(B, G * H, d, dtype=torch.bfloat16, device="cuda")
    q[-1] = small.q[0]
    kn, vn = (x.expand(B, H, d).contiguous() for x in (small.k_new, small.v_new))
    logc = torch.full((B, H, 1), -float("inf"), device="cuda")
    out = torch.empty(B, G * H, d, device="cuda")
    ws = torch.empty(rk.reskv_decode_quant_workspace_size(shape), dtype=torch.uint8, device="cuda")
    rk.reskv_decode_attn_quant(shape, rk.make_gate(), q, cache, logc, rl, ml, out, ws, k_new=kn, v_new=vn)
    want = small.decode({}, append=True)[0]
    K = torch.zeros(B, H, 1, d, dtype=torch.bfloat16, device="cuda")
    V = torch.zeros_like(K)
    rk.reskv_unpack_quant(shape, cache, rl, ml, K, V, first_slot=ml - 1)
    assert torch.equal(cache[-small.cache.numel():], small.cache)
    assert (host(K)[-1, :, 0] == ref.quantize(host(kn))[0][-1]).all()
    # the two shapes may take different kernels: the same sums in another order
    assert (out[-1] - want[0]).abs().max() <= 2.0 ** -15 * want.abs().max()


def test_graph_replays_match_eager_steps():
    """A captured step (rotation, append, decode) replayed with new inputs and eager steps between."""
    B, H, G, d, C = 2, 2, 4, 128, 700
    c = Case(17, "bf16", d, B, H, G, C, 64, [[3, 64], [0, 20]], [[1, 100], [600, 63]])
    plan, pos = rk.make_rope(d), i32([10, 20])
    caches, lens = [c.cache.clone(), c.cache.clone()], [c.main_len.clone(), c.main_len.clone()]
    outs = [torch.zeros(B, G * H, d, device="cuda") for _ in range(2)]
    wss = [torch.zeros(rk.reskv_decode_quant_workspace_size(c.shape), dtype=torch.uint8, device="cuda")
           for _ in range(2)]

    def call(i):
        rk.reskv_decode_attn_quant(c.shape, rk.make_gate(), c.q, caches[i], c.logc_dev, c.res_len, lens[i], outs[i],
                                   wss[i], rope=plan, positions=pos, k_new=c.k_new, v_new=c.v_new)

    call(0)
    lens[0].copy_(c.main_len)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(1)
    for step in range(6):
        c.q.copy_(dev(c.rng.normal(size=c.q.shape), "bf16"))
        c.k_new.copy_(dev(c.rng.normal(size=c.k_new.shape), "bf16"))
        pos.add_(1)
        torch.cuda.synchronize()
        g.replay()
        call(0)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.equal(lens[0], lens[1]) and torch.equal(caches[0], caches[1])
    assert (lens[0].cpu() == torch.minimum(c.main_len.cpu() + 6, C - c.res_len.cpu())).all()


def test_two_streams_at_once():
    """Two decodes on two streams with workspaces of their own."""
    cs = [Case(20 + i, "bf16", 128, 2, 4, 4, 3000, 300) for i in range(2)]
    want = [c.decode({}) for c in cs]
    streams = [torch.cuda.Stream() for _ in cs]
    outs = [torch.zeros_like(w[0]) for w in want]
    wss = [torch.empty(rk.reskv_decode_quant_workspace_size(c.shape), dtype=torch.uint8, device="cuda") for c in cs]
    torch.cuda.synchronize()
    for _ in range(5):
        for c, s, o, w in zip(cs, streams, outs, wss):
            rk.reskv_decode_attn_quant(c.shape, rk.make_gate(), c.q, c.cache, c.logc_dev, c.res_len, c.main_len, o, w,
                                       stream=s)
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert torch.equal(o, w[0])


def test_whole_run_from_prompt_to_steps():
    """As a user runs them: rotate a prompt's queries and keys out of token-major projections, build the compressed
    cache, pack it, then decode steps that rotate and append, with a follow-up chunk appended between. Every step is
    held to the oracle over the values read back, which are those of the kept rows and of the appended tokens."""
    rng = np.random.default_rng(30)
    B, Hq, H, d, S, w, budget, r = 2, 8, 2, 128, 700, 16, 128, 24
    C, Rcap = budget + 40, r
    shape = rk.make_shape(B, Hq, H, d, "bf16", C, Rcap)
    plan = rk.make_rope(d, scaling="llama3", theta=500000.0, factor=8.0, original_len=8192.0)

    def proj(n, heads):
        return dev(rng.normal(size=(B, n, heads, d)), "bf16").transpose(1, 2)

    pos = torch.arange(S, dtype=torch.int32, device="cuda").expand(B, S).contiguous()
    q, k, v = proj(S, Hq), proj(S, H), proj(S, H).contiguous()
    qr = torch.empty(B, Hq, w, d, dtype=torch.bfloat16, device="cuda")
    kr = torch.empty(B, H, S, d, dtype=torch.bfloat16, device="cuda")
    rk.reskv_rope(shape, plan, pos, k=k, k_out=kr)
    rk.reskv_rope(shape, plan, pos[:, S - w:].contiguous(), q=q[:, :, S - w:], q_out=qr)
    params = rk.BuildParams(S, w, w, 4, 0, 0)
    kc, vc = (torch.zeros(B, H, C, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    logc = torch.zeros(B, H, Rcap, device="cuda")
    idx = torch.zeros(B, H, C, dtype=torch.int32, device="cuda")
    rl, ml = i32(np.zeros(B * H)), i32(np.zeros(B * H))
    ws = torch.empty(rk.reskv_build_workspace_size(shape, params, [S] * B, [budget] * B, [r] * (B * H)),
                     dtype=torch.uint8, device="cuda")
    rk.reskv_build_cache(shape, params, kr, v, [S] * B, qr, [budget] * B, [r] * (B * H), kc, vc, logc, idx, rl, ml, ws)
    cache = torch.empty(rk.reskv_quant_cache_size(shape), dtype=torch.uint8, device="cuda")
    rk.reskv_pack_quant(shape, kc, vc, rl, ml, cache)
    K, V = ref.quantize(host(kc))[0], ref.quantize(host(vc))[0]
    dws = torch.empty(rk.reskv_decode_quant_workspace_size(shape), dtype=torch.uint8, device="cuda")
    c = Case.__new__(Case)
    c.B, c.H, c.G, c.d, c.r, c.logc = B, H, Hq // H, d, np.full((B, H), r), host(logc)
    n, at = np.full((B, H), budget - r), S
    for step in range(6):
        if step == 3:  # a follow-up of five tokens, three in the second sequence
            kn, vn = proj(5, H).contiguous(), proj(5, H).contiguous()
            p = torch.arange(at, at + 5, dtype=torch.int32, device="cuda").expand(B, 5).contiguous()
            rk.reskv_append_kv_quant(shape, kn, vn, cache, rl, ml, rope=plan, positions=p, n_tok=i32([5, 3]))
            turned = torch.empty_like(kn)
            rk.reskv_rope(shape, plan, p, k=kn, k_out=turned)
            for b, m in enumerate((5, 3)):
                for h in range(H):
                    K[b, h, r + n[b, h]:r + n[b, h] + m] = ref.quantize(host(turned)[b, h, :m])[0]
                    V[b, h, r + n[b, h]:r + n[b, h] + m] = ref.quantize(host(vn)[b, h, :m])[0]
                    n[b, h] += m
            at += 5
        qs, kn, vn = proj(1, Hq).contiguous(), proj(1, H).contiguous(), proj(1, H).contiguous()
        p = torch.full((B, 1), at, dtype=torch.int32, device="cuda")
        out = torch.empty(B, Hq, d, device="cuda")
        stats = [torch.empty(B * Hq, device="cuda") for _ in range(3)]
        rk.reskv_decode_attn_quant(shape, rk.make_gate(), qs, cache, logc, rl, ml, out, dws, rope=plan, positions=p,
                                   k_new=kn, v_new=vn, dbg_lse_main=stats[0], dbg_lse_res=stats[1], dbg_gate=stats[2])
        qt, kt = torch.empty_like(qs), torch.empty_like(kn)
        rk.reskv_rope(shape, plan, p, q=qs, q_out=qt, k=kn, k_out=kt)
        for b in range(B):
            for h in range(H):
                K[b, h, r + n[b, h]] = ref.quantize(host(kt)[b, h, 0])[0]
                V[b, h, r + n[b, h]] = ref.quantize(host(vn)[b, h, 0])[0]
        n, at = n + 1, at + 1
        assert (ml.cpu().numpy().reshape(B, H) == n).all()
        c.check([out] + [s.reshape(B, Hq) for s in stats], {}, q=host(qt)[:, :, 0], K=K, V=V, n=n)
    ko, vo = torch.zeros_like(kc), torch.zeros_like(vc)
    rk.reskv_unpack_quant(shape, cache, rl, ml, ko, vo)
    live = (np.arange(C) < (n + r)[..., None])[..., None]
    assert (host(ko) == np.where(live, K, 0)).all() and (host(vo) == np.where(live, V, 0)).all()
