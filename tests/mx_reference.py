"""Microscaling formats from their definition, with numpy: codes and scales of 32-bit
numbers, their values in 64 bits, and the keys as the append rounds them on the way."""
import math

import numpy as np
import torch

BLOCK = 32
# magnitudes by code
SIZES = {4: np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6]),
         8: np.array([m / 8 * 2.0 ** -6 for m in range(8)] +
                     [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8)][:-1])}
LIMIT = {4: 7.0, 8: 464.0}
MOST = {(torch.float16, 4): 49152.0, (torch.float16, 8): 61440.0}
for _t in (torch.bfloat16, torch.float32):
    MOST[_t, 4], MOST[_t, 8] = 6 * 2.0 ** 125, 15 * 2.0 ** 124


def encode(x, bits, dtype):
    """(codes, scales), bytes, of x [..., dim] whose elements are numbers of 32 bits at most."""
    dim = x.shape[-1]
    blocks = -(-dim // BLOCK)
    x = np.concatenate([x.astype(np.float64),
                        np.zeros((*x.shape[:-1], blocks * BLOCK - dim))], axis=-1)
    x = x.reshape(*x.shape[:-1], blocks, BLOCK)
    bad = ~np.isfinite(x).all(axis=-1)
    negative = np.signbit(x)
    size = np.minimum(np.abs(np.where(bad[..., None], 0, x)), MOST[dtype, bits])
    top = size.max(axis=-1)
    e = np.full(top.shape, -110)
    while (top > LIMIT[bits] * 2.0 ** e).any():
        e = np.where(top > LIMIT[bits] * 2.0 ** e, e + 1, e)
    y = size / 2.0 ** e[..., None]
    middles = (SIZES[bits][1:] + SIZES[bits][:-1]) / 2
    low, high = np.searchsorted(middles, y), np.searchsorted(middles, y, side="right")
    code = np.where(low % 2 == 0, low, high)   # they differ where y is in the middle
    code = np.where(bad[..., None], 0, code + (negative << (bits - 1)))
    code = code.reshape(*code.shape[:-2], blocks * BLOCK)
    if bits == 4:
        code = code[..., 0::2] | code[..., 1::2] << 4
    return code.astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def decode(codes, scales, dim):
    """Values in 64 bits."""
    bits = codes.shape[-1] // (4 * scales.shape[-1])
    if bits == 4:
        codes = np.stack([codes & 15, codes >> 4], axis=-1)
        codes = codes.reshape(*codes.shape[:-2], 2 * codes.shape[-2])
    sizes = np.append(SIZES[8], math.nan) if bits == 8 else SIZES[4]
    half = 1 << (bits - 1)
    x = np.where(codes >= half, -1.0, 1.0) * sizes[codes % half]
    scale = np.where(scales == 255, math.nan, 2.0 ** (scales.astype(np.int64) - 127))
    return (x * np.repeat(scale, BLOCK, axis=-1))[..., :dim]


def keys(k, w, cos, sin, interleaved, eps):
    """What the append holds keys' codes of, in 32 bits: k [tokens, heads, dim], w or None, cos and
    sin [tokens, rotary / 2] in 32 bits."""
    x = k.astype(np.float32)
    with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
        if w is not None:
            x64 = x.astype(np.float64)
            rstd = 1 / np.sqrt((x64 * x64).mean(axis=-1, keepdims=True) + np.float32(eps))
            x = x * rstd.astype(np.float32) * w.astype(np.float32)
        i = np.arange(cos.shape[-1])
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + cos.shape[-1])
        c, s = cos[:, None].astype(np.float32), sin[:, None].astype(np.float32)
        y = x.copy()
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y
