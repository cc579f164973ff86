"""Block-scaled low-bit formats, products of them, and gradients around them.

Test infrastructure: used only by tests.  fp64 throughout; every function
states the definition, with no regard to speed.
"""
from __future__ import annotations

import numpy as np

BLOCK = 32
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
# e4m3: eight subnormal steps of 2^-9, then 1.m * 2^e up to 448 (the pattern
# after it is the NaN).
E4M3 = np.array([i * 2.0 ** -9 for i in range(8)]
                + [(1 + i / 8) * 2.0 ** e for e in range(-6, 9) for i in range(8)][:-1])


def nearest_code(a, grid):
    """Index of the grid value nearest to a >= 0, ties to the even index,
    values past the end to the last."""
    a = np.minimum(np.asarray(a, np.float64), grid[-1])
    mid = (grid[1:] + grid[:-1]) / 2
    lo = np.searchsorted(mid, a, side="left")      # number of midpoints < a
    hi = np.searchsorted(mid, a, side="right")     # ... <= a
    return np.where(lo == hi, lo, np.where(lo % 2 == 0, lo, hi))


def _blocks(x):
    x = np.asarray(x, np.float64)
    n = -(-x.shape[1] // BLOCK)
    pad = np.zeros((x.shape[0], n * BLOCK))
    pad[:, :x.shape[1]] = x
    return pad.reshape(x.shape[0], n, BLOCK)


def block_exponents(x, bits: int):
    """Each block's scale exponent [M, ceil(K / 32)]; 128 marks a block that
    holds an infinity or a NaN.  4 bits: floor(log2 of the largest) - 2.  8 bits: the
    least e with largest / 2^e <= 448.  Not below -127."""
    v = np.abs(_blocks(x))
    with np.errstate(invalid="ignore"):
        bad = ~np.isfinite(v).all(axis=2)
        top = np.where(bad, 1.0, v.max(axis=2, initial=0.0))
    m, e = np.frexp(np.where(top > 0, top, 1.0))
    e = e - 1                                       # floor(log2)
    e = e - 2 if bits == 4 else e - 8 + (2 * m * 256 > 448)
    e = np.where(top > 0, np.maximum(e, -127), -127)
    return np.where(bad, 128, e)


def hold(x, bits: int):
    """(codes [M, K], exponents): what x is held as.  Code: sign bit above the
    magnitude's index in the format's grid (undefined in a marked block)."""
    grid = E2M1 if bits == 4 else E4M3
    e = block_exponents(x, bits)
    v = _blocks(x)
    with np.errstate(invalid="ignore", over="ignore"):
        a = np.where(e[..., None] == 128, 0.0, np.abs(v)) * 2.0 ** -np.where(e == 128, 0, e)[..., None].astype(np.float64)
    c = nearest_code(a, grid) + np.signbit(v) * (8 if bits == 4 else 128)
    return c.reshape(len(v), BLOCK * v.shape[1])[:, :np.shape(x)[1]].astype(np.uint8), e


def held_values(codes, e, bits: int):
    grid = E2M1 if bits == 4 else E4M3
    half = 8 if bits == 4 else 128
    v = grid[codes % half] * np.where(codes >= half, -1.0, 1.0)
    s = np.where(e == 128, np.nan, 2.0 ** np.where(e == 128, 0, e).astype(np.float64))
    return v * np.repeat(s, BLOCK, axis=1)[:, :codes.shape[1]]


def mx_pack(codes, e):
    """The 4-bit layout: two codes to a byte (the even column low), scales
    [ceil(K / 64), M rounded up to 8, 2] with zeros where nothing is held."""
    M, K = codes.shape
    s = np.zeros((-(-M // 8) * 8, -(-K // 64) * 2), np.uint8)
    s[:M, :K // BLOCK] = np.where(e == 128, 255, e + 127)
    return (codes[:, ::2] | codes[:, 1::2] << 4).astype(np.uint8), s.reshape(len(s), -1, 2).transpose(1, 0, 2).copy()


def mx_unpack(q, s):
    M, K = q.shape[0], 2 * q.shape[1]
    codes = np.empty((M, K), np.uint8)
    codes[:, ::2], codes[:, 1::2] = q & 15, q >> 4
    e = s.transpose(1, 0, 2).reshape(s.shape[1], -1)[:M, :K // BLOCK].astype(np.int64)
    return codes, np.where(e == 255, 128, e - 127)


def ckpt_scales(e):
    return np.where(e == 128, 255, e + 127).astype(np.uint8)


def image_rows(vec, off):
    """Per-image vectors [B, D] spread over the images' rows."""
    return np.repeat(np.asarray(vec, np.float64), np.diff(off), axis=0)


def norm_forward(x, shift, scale, off, eps):
    """h, mean, rstd of the modulated layer norm; shift, scale [B, D]."""
    x = np.asarray(x, np.float64)
    mean = x.mean(axis=1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(axis=1) + eps)
    n = (x - mean[:, None]) * rstd[:, None]
    return n * (1.0 + image_rows(scale, off)) + image_rows(shift, off), mean, rstd


def norm_backward(dh, x, mean, rstd, scale, off, dres=None):
    """dx, dscale [B, D], dshift [B, D] with mean and rstd as given."""
    dh, x = np.asarray(dh, np.float64), np.asarray(x, np.float64)
    n = (x - mean[:, None]) * rstd[:, None]
    g = dh * (1.0 + image_rows(scale, off))
    dx = rstd[:, None] * (g - g.mean(axis=1, keepdims=True) - n * (g * n).mean(axis=1, keepdims=True))
    if dres is not None:
        dx = dx + dres
    parts = [slice(a, b) for a, b in zip(off, off[1:])]
    return dx, np.stack([(dh * n)[p].sum(axis=0) for p in parts]), np.stack([dh[p].sum(axis=0) for p in parts])


def gelu_slope(x):
    """Derivative of the tanh GELU through the logistic s of 2u (1 + tanh u
    would keep no digits far below zero)."""
    x = np.asarray(x, np.float64)
    u2 = 2.0 * np.sqrt(2.0 / np.pi) * (x + 0.044715 * x ** 3)
    e = np.exp(-np.abs(u2))
    s = np.where(u2 >= 0, 1.0, e) / (1.0 + e)
    return s + x * (e / (1.0 + e) ** 2) * 2.0 * np.sqrt(2.0 / np.pi) * (1.0 + 3 * 0.044715 * x ** 2)
