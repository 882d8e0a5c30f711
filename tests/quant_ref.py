"""Plain implementations, in 64 bits, of what the rotary positions and the 4-bit
caches are held to: the format from its definition (a search over the sixteen
values), the buffer layout by its index formulas, the rotation pair by pair.
Nothing here is shared with the library."""

import math

import numpy as np

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantize(x):
    """Rows x [..., d] as (values they stand for, codes, scale bytes [..., d/32])."""
    x = np.asarray(x, np.float64)
    g = x.reshape(*x.shape[:-1], -1, 32)
    amax = np.abs(g).max(-1)
    bad = ~np.isfinite(amax)
    e = np.full(amax.shape, -125)
    for k in range(-125, 125):  # the least power of two that no magnitude passes seven times
        e += np.where(bad, 0.0, amax) > 7.0 * 2.0 ** k
    with np.errstate(invalid="ignore"):
        y = np.abs(g) / 2.0 ** e[..., None].astype(np.float64)
        dist = np.abs(np.minimum(np.where(np.isfinite(y), y, 0.0), 6.0)[..., None] - VALUES)
    near = dist == dist.min(-1, keepdims=True)
    first, last = near.argmax(-1), 7 - near[..., ::-1].argmax(-1)
    code = np.where(first % 2 == 0, first, last)  # ties to the even code
    sign = np.signbit(g)
    value = np.where(sign, -1.0, 1.0) * VALUES[code] * 2.0 ** e[..., None].astype(np.float64)
    value = np.where(bad[..., None], np.nan, value)
    byte = np.where(bad, 255, e + 127)
    return value.reshape(x.shape), (code + 8 * sign).reshape(x.shape).astype(np.uint8), byte.astype(np.uint8)


def places(d, C):
    """Byte offsets in a (b, kv head) buffer of every slot's key and value codes [C, d] and scales [C, d/32]."""
    s_all, i, c = np.arange(C)[:, None], np.arange(d)[None], np.arange(d // 32)[None]
    base, s, P = (s_all // 64) * 68 * d, s_all % 64, d // 16
    return (base + s * (d // 2) + i // 2,
            base + 32 * d + ((s // 4) * 16 + i // P) * 2 * P + (s % 4) * (P // 2) + (i % P) // 2,
            base + 64 * d + ((s % 16) * (d // 32) + c) * 4 + s // 16,
            base + 66 * d + ((((s // 4) % 4) * (d // 32) + c) * 4 + s // 16) * 4 + s % 4)


def pack(K, V, live, fill=0):
    """[B*H, bytes] buffer of K, V [B, H, C, d] with `live` [B, H] slots each; other bytes `fill`."""
    B, H, C, d = K.shape
    nb = -(-C // 64)
    buf = np.full((B * H, nb * 68 * d), fill, np.uint8)
    pk, pv, sk, sv = places(d, C)
    for x, pc, ps in ((K, pk, sk), (V, pv, sv)):
        _, code, byte = quantize(x)
        code, byte = code.reshape(B * H, C, d), byte.reshape(B * H, C, d // 32)
        for bh in range(B * H):
            n = int(np.asarray(live).reshape(-1)[bh])
            buf[bh, pc[:n, 0::2]] = code[bh, :n, 0::2] + 16 * code[bh, :n, 1::2]
            buf[bh, ps[:n]] = byte[bh, :n]
    return buf


def frequencies(rot, theta=10000.0, scaling="none", factor=1.0, original_len=0.0, low_freq_factor=1.0,
                high_freq_factor=4.0, beta_fast=32.0, beta_slow=1.0, attn_scale=0.0, **_):
    """(radians a position [rot/2], factor on rotated pairs)."""
    out, scale = [], attn_scale or (0.1 * math.log(factor) + 1.0 if scaling == "yarn" else 1.0)
    for i in range(rot // 2):
        base = theta * factor ** (rot / (rot - 2.0)) if scaling == "ntk" else theta
        f = base ** (-2.0 * i / rot)
        if scaling == "linear":
            f /= factor
        if scaling == "llama3":
            wave = 2.0 * math.pi / f
            if wave > original_len / low_freq_factor:
                f /= factor
            elif wave >= original_len / high_freq_factor:
                t = (original_len / wave - low_freq_factor) / (high_freq_factor - low_freq_factor)
                f = (1.0 - t) * f / factor + t * f
        if scaling == "yarn":
            lo, hi = (rot * math.log(original_len / (2.0 * math.pi * b)) / (2.0 * math.log(theta))
                      for b in (beta_fast, beta_slow))
            lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), rot - 1)
            t = min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0)
            f = (1.0 - t) * f + t * f / factor
        out.append(f)
    return np.array(out), scale


def rotate(x, pos, rot, layout="half", **kw):
    """Rows x [B, heads, n, d] at positions pos [B, n], in 64 bits, unrounded."""
    x = np.array(x, np.float64)
    f, scale = frequencies(rot, **kw)
    a = np.asarray(pos, np.float64)[:, None, :, None] * f
    c, s = scale * np.cos(a), scale * np.sin(a)
    i = np.arange(rot // 2)
    p, q = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
    u, v = x[..., p], x[..., q]
    x[..., p], x[..., q] = u * c - v * s, u * s + v * c
    return x


def rotate_atol(x, pos, rot, eps, layout="half", **kw):
    """Bound on |rotate(x) rounded to a type of this eps - rotate(x)|: half a step of the result (eps / 2 of it),
    and the error of the angle in 64 bits: the frequency's and the product's rounding (three of 2^-53 relative on
    either side, six in all) times the pair's length, and a few 2^-52 of the pair from sines and products."""
    ref = rotate(x, pos, rot, layout, **kw)
    f, scale = frequencies(rot, **kw)
    angle = np.abs(np.asarray(pos, np.float64))[:, None, :, None] * f
    i = np.arange(rot // 2)
    p, q = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
    x = np.asarray(x, np.float64)
    length = np.abs(x[..., p]) + np.abs(x[..., q])
    slack = np.zeros(x.shape)
    slack[..., p] = slack[..., q] = scale * length * (angle * 6 * 2.0 ** -53 + 8 * 2.0 ** -52)
    return ref, np.abs(ref) * eps / 2 + slack * (1 + eps)


def decode_atol(q, K, V, gate, lse_main, alpha, g_min):
    """Bound on the error of one query's output. A logit is an fp32 sum of d exact products (three bf16 parts of
    an fp32 query make 3 d), scaled once and fed to a base-2 exponential of a few ulp: off by at most
    delta = (3 d + 8) u max sum |q_i k_i| / sqrt(d) + 2^-20, u = 2^-24, so every weight is off by e^delta - 1 relative
    and a weighted mean by twice that of the largest value. The probabilities enter as two bf16 parts, each rounded
    to nearest: 2^-18 relative; the sums of n terms and the merge of 8 states in fp32: (n / 8 + 64) u. The gate moves
    the residual part: its relative error (as delta moves p_max, slope alpha (1 - g)) of the largest value."""
    q, K, V = (np.asarray(t, np.float64) for t in (q, K, V))
    d = q.shape[-1]
    mag = float((np.abs(K) @ np.abs(q)).max()) / np.sqrt(d) if len(K) else 0.0
    delta = (3 * d + 8) * 2.0 ** -24 * mag + 2.0 ** -20
    rel = 2.0 * np.expm1(2.0 * delta) + 2.0 ** -17 + (len(K) / 8 + 64) * 2.0 ** -24
    g_rel = alpha * (1.0 - min(gate, 1.0)) * np.expm1(2.0 * delta) if gate > g_min else 0.0
    return (rel + g_rel) * float(np.abs(V).max(initial=0.0))
