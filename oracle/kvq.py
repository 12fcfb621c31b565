"""A key/value cache held in 4 bits, by its definition, in 64 bits (numpy).

Blocks of 32 consecutive head-dim elements share 2^e, e the smallest integer with max|x| < 7 * 2^e within [-124, 125]; an
element is the nearest of 0, .5, 1, 1.5, 2, 3, 4, 6 times 2^e (ties to the even code, at most 6) with its sign; the scale
is stored as the byte e + 127, and a block with a value that is not finite as 255 with codes of 0."""
from __future__ import annotations

import numpy as np

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise(x):
    """x [..., dh] -> codes uint8 [..., dh / 2], scales uint8 [..., dh / 32]."""
    x = np.asarray(x, np.float64)
    x = x.reshape(*x.shape[:-1], -1, 32)
    top = np.abs(x).max(-1)                                   # NaN where the block holds one
    fine = np.isfinite(top)
    # candidates from below: the first e that satisfies the definition
    e = np.full(top.shape, -124)
    guess = np.floor(np.log2(np.where(fine & (top > 0), top, 1.0) / 8.0)).astype(int) - 1
    for step in range(4):
        unmet = fine & (top >= 7.0 * 2.0 ** e)
        e = np.where(unmet, np.clip(guess + step, -124, 125), e)
    y = np.where(fine[..., None], x / 2.0 ** e[..., None], 0.0)
    mag = np.minimum(np.abs(y), 6.0)
    # nearest value; among two equally near ones the even code, which comes first in this order
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])
    code = order[np.abs(mag[..., None] - VALUES[order]).argmin(-1)].astype(np.uint8)
    code = np.where(fine[..., None], code | (np.signbit(y).astype(np.uint8) << 3), 0).astype(np.uint8)
    code = code.reshape(*code.shape[:-2], -1)
    return code[..., 0::2] | (code[..., 1::2] << 4), np.where(fine, e + 127, 255).astype(np.uint8)


def values(codes, scales):
    """What codes [..., dh / 2] and scales [..., dh / 32] stand for."""
    c = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1)
    x = np.where(c & 8, -1.0, 1.0) * VALUES[c & 7]
    size = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return x * np.repeat(size, 32, axis=-1)


def attention(q, k, v, scale, lens, mask=None):
    """q [B,n,H,dh], k and v [B,heads,L,dh] (values), lens [B], mask [B,L] or None -> [B,n,H,dh]."""
    B, n, H, dh = q.shape
    group = H // k.shape[1]
    out = np.zeros(q.shape, np.float64)
    for b in range(B):
        seen = np.arange(k.shape[2]) < lens[b]
        if mask is not None:
            seen &= mask[b] != 0
        if not seen.any():
            continue
        for h in range(H):
            kk, vv = k[b, h // group, seen], v[b, h // group, seen]
            s = scale * (q[b, :, h].astype(np.float64) @ kk.T)
            p = np.exp(s - s.max(-1, keepdims=True))
            out[b, :, h] = p @ vv / p.sum(-1, keepdims=True)
    return out
