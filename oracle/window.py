"""Attention with a sliding window and sinks, and the KV cache of 4 bits, in float64 from their definitions.  TEST INFRASTRUCTURE ONLY.

The query at position i sees key j where j <= i and (j > i - window or j < sinks).

Cache of 4 bits: 64 consecutive values share a scale s and a center c, both IEEE half, s = half((hi - lo) (1/15)) and
c = half(lo + 8 s) with float32 operations; a value is held as the nearest c + s u, u whole in -8 .. 7 (the even u half way).
A page holds 16 tokens; per KV head: K codes, V codes, (s, c) of K, (s, c) of V.
"""
import numpy as np


def visible(q_pos, n_keys, window, sinks):
    """[T, n_keys] of bool."""
    i, j = np.asarray(q_pos, np.int64)[:, None], np.arange(n_keys)[None, :]
    return (j <= i) & ((j > i - window) | (j < sinks))


def attention(q, k, v, q_pos, window, sinks):
    """q [T, Hq, hd] at positions q_pos, k, v [S, Hkv, hd]: outputs [T, Hq, hd].  Keys that a query does not see take no part,
    whatever they hold."""
    T, Hq, hd = q.shape
    S, Hkv, _ = k.shape
    see = visible(q_pos, S, window, sinks)
    out = np.empty((T, Hq, hd))
    for t in range(T):
        at = np.flatnonzero(see[t])
        for h in range(Hq):
            kk, vv = k[at, h // (Hq // Hkv)], v[at, h // (Hq // Hkv)]
            with np.errstate(all="ignore"):
                z = kk @ q[t, h] / np.sqrt(hd)
                p = np.exp(z - z.max())
                out[t, h] = (p / p.sum()) @ vv
    return out


# ---------------------------------------------------------------------------------------------------- cache of 4 bits

def kv4_quantize(x):
    """x [..., hd]: codes u + 8 (uint8, [..., hd]) and parameters (s, c) as float16 [..., hd / 64, 2]."""
    x = np.asarray(x)
    g = x.reshape(*x.shape[:-1], x.shape[-1] // 64, 64)
    with np.errstate(all="ignore"):
        f = g.astype(np.float32)
        lo, hi = f.min(-1), f.max(-1)
        s = (np.subtract(hi, lo, dtype=np.float32) * np.float32(np.float32(1) / np.float32(15))).astype(np.float16)
        c = (lo + np.float32(8) * s.astype(np.float32)).astype(np.float16)
        bad = ~(np.abs(g) <= 65504).all(-1)
        s, c = np.where(bad, np.float16(np.nan), s), np.where(bad, np.float16(np.nan), c)
        step = s.astype(np.float64)[..., None]
        u = np.rint((g.astype(np.float64) - c.astype(np.float64)[..., None]) / np.where(step > 0, step, 1.0))
        u = np.where(step > 0, np.clip(u, -8, 7), 0.0)
    return (u + 8).astype(np.uint8).reshape(x.shape), np.stack([s, c], -1)


def kv4_values(codes, params):
    u = codes.reshape(*codes.shape[:-1], codes.shape[-1] // 64, 64).astype(np.float64) - 8
    p = params.astype(np.float64)
    return (p[..., 1:2] + p[..., 0:1] * u).reshape(codes.shape)


def kv4_round(x):
    """What the cache holds for x."""
    return kv4_values(*kv4_quantize(x))


def kv4_places(hd):
    """Byte and bit in a block of the codes of K and V of (token, dim), and the byte of the (s, c) pair of K: five arrays [16, hd]."""
    t, d = np.arange(16)[:, None], np.arange(hd)[None, :]
    a, w = d // 32, hd // 32
    b, i = d % 32 // 8, d % 8
    k_byte, k_bit = ((16 * b + t) * w + a) * 4 + i // 2, 4 * (i % 2) + 0 * t
    e, g = d % 32 // 16, d % 16
    v_byte, v_bit = 8 * hd + ((16 * (t // 4) + g) * w + a) * 4 + t % 4, 4 * e + 0 * t
    return k_byte, k_bit, v_byte, v_bit, 16 * hd + (d // 64 * 16 + t) * 4


def kv4_write(block, token, k, v):
    """One token's K and V [hd] into a block (uint8 [18 hd])."""
    hd = len(k)
    k_byte, k_bit, v_byte, v_bit, par = kv4_places(hd)
    for x, byte, bit, at in ((k, k_byte, k_bit, 0), (v, v_byte, v_bit, hd)):
        codes, params = kv4_quantize(x)
        for d in range(hd):
            B, s = byte[token, d], int(bit[token, d])
            block[B] = (int(block[B]) & ~(15 << s) & 255) | int(codes[d]) << s
        for g in range(hd // 64):
            p = at + par[token, 64 * g]
            block[p:p + 4] = params[g].view(np.uint8)


def kv4_block_values(block, hd):
    """K and V [16, hd] that a block holds."""
    k_byte, k_bit, v_byte, v_bit, par = kv4_places(hd)
    out = []
    for byte, bit, at in ((k_byte, k_bit, 0), (v_byte, v_bit, hd)):
        u = (block[byte] >> bit) % 16
        half = np.ascontiguousarray(block).view(np.float16).astype(np.float64)
        p = (at + par) // 2
        out.append(half[p + 1] + half[p] * (u - 8.0))
    return out
