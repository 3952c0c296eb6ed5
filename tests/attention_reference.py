"""The operators of one device's share of an attention block from their
definitions, in 64 bits with numpy, and bounds on what 32-bit sums and one
rounding may be off by."""
import math

import numpy as np
import torch

ROUND = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
# half the distance between the smallest values of a type
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}
E32 = 2.0 ** -24


def f64(t):
    return t.detach().cpu().double().numpy()


def pairs(dim, rotary, interleaved):
    """Index pairs (a, b) of the rotation."""
    i = np.arange(rotary // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)


def rotate(x, cos, sin, interleaved, back=False):
    """x [..., dim] by angles [..., rotary / 2] (broadcast over heads by the caller)."""
    a, b = pairs(x.shape[-1], 2 * cos.shape[-1], interleaved)
    y = x.copy()
    s = -sin if back else sin
    y[..., a] = x[..., a] * cos - x[..., b] * s
    y[..., b] = x[..., b] * cos + x[..., a] * s
    return y


def spread(x, rotary, interleaved):
    """|x_a| + |x_b| for both members of every pair: what a rotation's terms add up to."""
    a, b = pairs(x.shape[-1], rotary, interleaved)
    m = np.abs(x)
    y = m.copy()
    y[..., a] = y[..., b] = m[..., a] + m[..., b]
    return y


def norm(x, w, eps):
    rstd = 1 / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps)
    return x * rstd * w, rstd


def norm_rotate(x, w, cos, sin, interleaved, eps, dtype):
    """(y, bound) for x [..., heads, dim]; w None: no norm; cos, sin [..., rotary / 2] per token."""
    n = x if w is None else norm(x, w, eps)[0]
    y = rotate(n, cos[..., None, :], sin[..., None, :], interleaved)
    # the mean's sum of dim squares, its root, three products and a sum
    bound = (x.shape[-1] + 16) * E32 * spread(n, 2 * cos.shape[-1], interleaved)
    return y, bound + ROUND[dtype] * (np.abs(y) + bound) + TINY[dtype]


def norm_rotate_gradients(g, x, w, cos, sin, interleaved, eps, dtype, weight_dtype):
    """(dx, its bound, dw, its bound)."""
    dim, rotary = x.shape[-1], 2 * cos.shape[-1]
    h = rotate(g, cos[..., None, :], sin[..., None, :], interleaved, back=True)
    size = spread(g, rotary, interleaved)
    if w is None:
        bound = 16 * E32 * size
        return h, bound + ROUND[dtype] * (np.abs(h) + bound) + TINY[dtype], None, None
    _, rstd = norm(x, w, eps)
    xh = x * rstd
    dx = rstd * (h * w - xh * (h * w * xh).mean(axis=-1, keepdims=True))
    terms = rstd * (size * np.abs(w) + np.abs(xh) *
                    (size * np.abs(w * xh)).mean(axis=-1, keepdims=True))
    bound = (3 * dim + 32) * E32 * terms
    rows = int(np.prod(x.shape[:-1]))
    axes = tuple(range(x.ndim - 1))
    dw = (h * xh).sum(axis=axes)
    dw_bound = (rows + dim + 32) * E32 * (size * np.abs(xh)).sum(axis=axes)
    return (dx, bound + ROUND[dtype] * (np.abs(dx) + bound) + TINY[dtype], dw,
            dw_bound + ROUND[weight_dtype] * (np.abs(dw) + dw_bound) + TINY[weight_dtype])


def attend(q, keys, values, first_pos, start, causal, window, scale, dtype):
    """q [tokens, q_heads, dim], keys and values [kv_len, kv_heads, dim] of one
    sequence: (out, bound, lse, its bound).  Only what a token sees is touched."""
    tokens, q_heads, dim = q.shape
    kv_len, kv_heads = keys.shape[:2]
    out = np.zeros_like(q)
    bound = np.zeros_like(q)
    lse = np.full((tokens, q_heads), -math.inf)
    lse_bound = np.zeros((tokens, q_heads))
    for t in range(tokens):
        lo, hi = start, kv_len
        if causal:
            hi = min(hi, first_pos + t + 1)
            if window:
                lo = max(lo, first_pos + t + 1 - window)
        if hi <= lo:
            continue
        for h in range(q_heads):
            k, v = keys[lo:hi, h // (q_heads // kv_heads)], values[lo:hi, h // (q_heads // kv_heads)]
            s = (k @ q[t, h]) * scale
            size = (np.abs(k) @ np.abs(q[t, h])) * scale
            m = s.max()
            p = np.exp(s - m)
            total = p.sum()
            out[t, h] = p @ v / total
            lse[t, h] = m + math.log(total)
            # a score's sum of dim products, its scaling and the exponent's shift; numerator and
            # denominator both; the sums over the keys, the joins' factors
            off = 2 * (2 * dim + 8) * E32 * size.max() + (2 * len(p) + 64) * E32
            weights = p @ np.abs(v) / total
            # numerators rounded to the type, those below its range to a multiple of its step
            # (the largest numerator is 1 or more)
            lost = TINY[dtype] * np.abs(v).sum(axis=0)
            b = (off + ROUND[dtype]) * weights + lost
            bound[t, h] = b + ROUND[dtype] * (np.abs(out[t, h]) + b) + TINY[dtype]
            lse_bound[t, h] = off + 4 * E32 * (abs(m) + abs(lse[t, h]) + 1)
    return out, bound, lse, lse_bound


def check(got, want, bound, what):
    got = f64(got) if isinstance(got, torch.Tensor) else got
    assert got.shape == want.shape, (what, got.shape, want.shape)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        off = np.where(same, 0, np.abs(got - want))
    bad = ~(off <= bound)
    if bad.any():
        at = np.argwhere(bad)[0]
        raise AssertionError(f"{what}: {bad.sum()} of {bad.size} values are off; first at "
                             f"{tuple(at)}: {got[tuple(at)]} for {want[tuple(at)]}, "
                             f"bound {bound[tuple(at)]}")
