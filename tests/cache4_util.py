"""Plain numpy forms of the 4-bit value cache, the key codes' values and attention over
them (64-bit sums), written from the definitions in include/pot_attn.h."""
from __future__ import annotations

import numpy as np

import oracle

GROUP = 288


def quantise4(v16):
    """fp16 rows [..., 64] to (n uint8 [..., 64], s, z fp16 [...])."""
    with np.errstate(all="ignore"):
        x = v16.astype(np.float32)
        x = np.where(np.isnan(x), x, np.clip(x, -65504, 65504))
        nan = np.isnan(x)
        none = nan.all(-1)
        z = np.where(none, 0, np.where(nan, np.inf, x).min(-1)).astype(np.float32)
        hi = np.where(none, 0, np.where(nan, -np.inf, x).max(-1)).astype(np.float32)
        f = ((hi - z).astype(np.float32) / np.float32(15)).astype(np.float32)
        s = f.astype(np.float16)
        low = s.astype(np.float32) < f
        s = np.where(low, (s.view(np.uint16) + 1).astype(np.uint16), s.view(np.uint16)).view(np.float16)
        inv = np.where(s > 0, np.float32(1) / s.astype(np.float32), 0).astype(np.float32)
        n = np.rint(((x - z[..., None]).astype(np.float32) * inv[..., None]).astype(np.float32))
        n = np.where(nan, 0, np.minimum(n, 15))
    return n.astype(np.uint8), s, z.astype(np.float16)


def dequantise4(n, s, z):
    """fp64 values."""
    return z.astype(np.float64)[..., None] + s.astype(np.float64)[..., None] * n


def place4(cache, n, s, z, t0):
    """Writes tokens t0 .. of every sequence into cache [n_seq, t_cap / 8, 288]; n [n_seq, n_tok, 64]."""
    c = np.arange(64)
    for i in range(n.shape[1]):
        g, u = divmod(t0 + i, 8)
        for half in (0, 1):
            lo, up = n[:, i, 32 * half:32 * half + 16], n[:, i, 32 * half + 16:32 * half + 32]
            cache[:, g, 16 * c[:16] + 8 * half + u] = lo | (up << 4)
        cache[:, g, 256:272].view(np.float16)[:, u] = s[:, i]
        cache[:, g, 272:288].view(np.float16)[:, u] = z[:, i]


def take4(cache):
    """fp64 values [n_seq, t_cap, 64] of a cache [n_seq, t_cap / 8, 288]."""
    c = np.arange(64)
    b = cache[:, :, (16 * (c % 16) + 8 * (c // 32))[None, :] + np.arange(8)[:, None]]
    n = np.where(c % 32 < 16, b & 15, b >> 4).astype(np.float64)
    s = np.ascontiguousarray(cache[:, :, 256:272]).view(np.float16).astype(np.float64)
    z = np.ascontiguousarray(cache[:, :, 272:288]).view(np.float16).astype(np.float64)
    v = z[..., None] + s[..., None] * n
    return v.reshape(cache.shape[0], -1, 64)


def key_values(se, cm, sc, k):
    """fp64 rows [rows, 64] that codes stand for, in the domain they were encoded in."""
    f = np.stack((se & 15, se >> 4), -1).reshape(se.shape[0], 64)
    j = np.zeros(f.shape)
    for b in range(k):
        bits = (cm[:, 8 * b:8 * b + 8, None] >> np.arange(8)) & 1
        j += bits.reshape(f.shape) * 2.0 ** (b - k)
    w = np.where(f & 8, -1.0, 1.0) * (1 + j) * 2.0 ** -(f & 7).astype(np.float64)
    with np.errstate(invalid="ignore"):
        return np.where((f & 7) == 7, 0.0, w * sc.astype(np.float64)[:, None])


def sylvester():
    h = np.ones((1, 1))
    for _ in range(6):
        h = np.block([[h, h], [h, -h]])
    return h


def attend(q, keys, values, lens, heads, hadamard):
    """fp64 attention with the quantised queries. keys, values [B, Hkv, rows, 64]. Returns O and the largest
    |score| in the log2 domain."""
    B, Hq, _ = q.shape
    qh, delta, _ = oracle.quantize_query(q, hadamard=hadamard)
    out = np.zeros((B, Hq, 64))
    top = 0.0
    for b in range(B):
        n = int(lens[b])
        if n == 0:
            continue
        for h in range(Hq):
            kv = heads[h]
            x = keys[b, kv, :n] @ qh[b, h].astype(np.float64) * (float(delta[b, h]) / 8)
            top = max(top, float(np.abs(x).max()) / np.log(2))
            p = np.exp(x - x.max())
            out[b, h] = p @ values[b, kv, :n] / p.sum()
    return out, top


def attend_bound(top, vmax, T):
    """Bound on |O - O64|. A score is made with at most 6 roundings of half a unit (query step, log2 e, the two
    products and the row scale's): 6 2^-24 |x| in its exponent, ln 2 of that in a weight, twice (sums and
    denominator): under 2^-20 |x|. A weight's exp2 and its fp16 parts: 2^-21 each, twice; the fp32 sums of T terms in
    chains of at most T / 64 + 64: T 2^-30 + 2^-18."""
    return vmax * (top * 2.0 ** -20 + 2.0 ** -19 + T * 2.0 ** -30 + 2.0 ** -18)
