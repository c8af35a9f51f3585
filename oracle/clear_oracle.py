"""Oracle of the clear track, float64 on the CPU: 4-bit weights, the 4-bit K/V format and attention, from their definitions.

No code is shared with the HIP kernels or with the packed layouts; matrices are plain float64 arrays.
"""
from __future__ import annotations

import numpy as np

GROUP = 32      # channels of a key or value that share a scale and an offset


def round_bf16(x):
    """float64 -> the nearest bfloat16 through float32, both to nearest even, as float64. NaN stays NaN."""
    f = np.asarray(x, np.float64).astype(np.float32)
    bits = f.view(np.uint32).astype(np.uint64)
    kept = ((bits + 0x7FFF + ((bits >> 16) & 1)) >> 16 << 16).astype(np.uint32)
    out = kept.view(np.float32).astype(np.float64)
    return np.where(np.isnan(f), np.nan, out)


def weights(codes, scales, offsets, K, group):
    """[M][K] float64 from packed codes ([M][(K+1)//2] uint8, even k in the low half) and group scales and offsets."""
    codes = np.asarray(codes)
    c = np.empty((codes.shape[0], 2 * codes.shape[1]), np.float64)
    c[:, 0::2] = codes & 15
    c[:, 1::2] = codes >> 4
    at = np.arange(K) // group
    w = np.asarray(scales, np.float64)[:, at] * (c[:, :K] - 8.0)
    return w if offsets is None else w + np.asarray(offsets, np.float64)[:, at]


def silu(a):
    return a / (1.0 + np.exp(-a))


def quantise(x):
    """(codes, scales, offsets) of [..][D]: codes [..][D] in 0..15, scales and offsets [..][D/32]."""
    g = np.asarray(x, np.float64)
    g = g.reshape(g.shape[:-1] + (g.shape[-1] // GROUP, GROUP))
    with np.errstate(all="ignore"):
        low, high = g.min(-1), g.max(-1)
        s = round_bf16((high - low) / 15.0)
        s = np.where(s >= 2.0 ** -126, s, 0.0)
        b = round_bf16(low - 16.0 * s)
        bad = ~np.isfinite(g).all(-1) | ~np.isfinite(s) | ~np.isfinite(b)
        s, b = np.where(bad, 0.0, s), np.where(bad, np.nan, b)
        c = np.clip(np.rint((g - b[..., None]) / s[..., None]) - 16.0, 0.0, 15.0)
    c = np.where((s > 0)[..., None], c, 0.0)
    return c.reshape(np.shape(x)).astype(np.int64), s, b


def held(x):
    """The values that the cache keeps of [..][D]."""
    c, s, b = quantise(x)
    return np.repeat(s, GROUP, -1) * (16.0 + c) + np.repeat(b, GROUP, -1)


def attention(q, k, v, scale, causal):
    """q [T][Hq][D] over k, v [L][Hkv][D]: row i sits at token L - T + i. A row that attends to nothing is zero; a token that a
    row does not attend to has no part in it, whatever it holds."""
    T, Hq, _ = q.shape
    L, Hkv, _ = k.shape
    out = np.zeros(q.shape, np.float64)
    for i in range(T):
        n = min(L, L - T + i + 1) if causal else L
        if n <= 0:
            continue
        for h in range(Hq):
            s = k[:n, h // (Hq // Hkv)] @ q[i, h] * scale
            p = np.exp(s - s.max())
            out[i, h] = (p / p.sum()) @ v[:n, h // (Hq // Hkv)]
    return out
