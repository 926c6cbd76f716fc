"""The microscaled 4-bit format and the norm in front of it, in numpy: what the tests hold the
kernels to.  Codes and exponents come from comparisons in 64 bits, not from the kernels'
conversions."""
from __future__ import annotations

import numpy as np

MAGNITUDES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def quantize(x):
    """x [T, K] (f32 or f64 values) -> codes uint8 [T, K], exponent bytes [T, ceil(K / 32)]."""
    T, K = x.shape
    nb = (K + 31) // 32
    b = np.zeros((T, nb * 32))
    b[:, :K] = x
    b = b.reshape(T, nb, 32)
    with np.errstate(invalid="ignore"):
        m = np.abs(b).max(-1)
        bad = ~(m < np.inf)
        m = np.where(bad, 1, m)
    e = np.where(m > 0, np.frexp(np.where(m > 0, m, 1))[1] - 1 - 2, -127)
    e = np.maximum(e, -127)
    u = np.ldexp(np.where(bad[..., None], 0, b), -e[..., None])
    a = np.abs(u)
    # between neighbours, a tie to the even code
    codes = np.zeros(a.shape, dtype=np.uint8)
    for c in range(1, 8):
        mid = (MAGNITUDES[c - 1] + MAGNITUDES[c]) / 2
        codes += ((a > mid) | ((a == mid) & (c % 2 == 0))).astype(np.uint8)
    codes += np.where(np.signbit(u) & ~bad[..., None], 8, 0).astype(np.uint8)
    return codes.reshape(T, -1)[:, :K], np.where(bad, 255, e + 127).astype(np.uint8)


def decode(codes, e):
    """Codes [T, K] and exponent bytes -> values in 64 bits (NaN in NaN blocks)."""
    T, K = codes.shape
    v = MAGNITUDES[codes & 7] * np.where(codes & 8, -1, 1)
    top = np.ldexp(1.0, np.where(e == 255, 0, e.astype(int) - 127))
    top = np.where(e == 255, np.nan, top)
    return v * np.repeat(top, 32, axis=1)[:, :K]


def pack(codes):
    """Codes [T, K] -> bytes [T, 16 ceil(K / 32)]."""
    T, K = codes.shape
    c = np.zeros((T, (K + 31) // 32 * 32), dtype=np.uint8)
    c[:, :K] = codes
    return c[:, 0::2] | (c[:, 1::2] << 4)


def tiles(e, K, fill=0):
    """Exponent bytes [T, ceil(K / 32)] -> the tiles of psc_mx4.h; fill: rows past T."""
    T, nb = e.shape
    n = (K + 127) // 128
    out = np.full((T + 127) // 128 * n * 512, fill, dtype=np.uint8)
    r, b = np.meshgrid(np.arange(T), np.arange(n * 4), indexing="ij")
    full = np.zeros((T, n * 4), dtype=np.uint8)
    full[:, :nb] = e
    out[512 * ((r // 128) * n + b // 4) + 16 * (r % 32) + 4 * (r % 128 // 32) + b % 4] = full
    return out


def norm(x, residual, gain, eps, bf16):
    """h (as f32, rounded as the stream holds it), v = h * gain in f32, r in 64 bits."""
    h = x.astype(np.float32)
    if residual is not None:
        with np.errstate(over="ignore", invalid="ignore"):
            h = h + residual.astype(np.float32)
        if bf16:
            h = round_bf16(h)
    g = np.ones(x.shape[1], dtype=np.float32) if gain is None else gain.astype(np.float32)
    with np.errstate(over="ignore", invalid="ignore"):
        v = h * g[None]
        r = 1 / np.sqrt((h.astype(np.float64) ** 2).mean(1) + eps)
    return h, v, r


def round_bf16(x):
    """f32 values rounded to bf16, ties to even (infinities and NaN stay)."""
    w = x.astype(np.float32).view(np.uint32)
    near = ((w.astype(np.uint64) + 0x7fff + ((w >> 16) & 1)) & 0xffff0000).astype(np.uint32)
    return np.where(np.isfinite(x), near, w).astype(np.uint32).view(np.float32)
