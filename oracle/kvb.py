"""A key/value cache held in 8 bits, by its definition, in 64 bits (numpy).

An element is an E4M3 number times 2^e, e the smallest integer within [-117, 119] with max|x| <= 464 * 2^e over the finite elements of a
block of 32 consecutive rows of one head, the nearest one (ties to the even code, at most 448) with its sign; what is not finite has
the code 127.  The scale is stored as the byte e + 127.  Rows written into a block that holds some raise its e where they have to, and the
rows held are then rounded to the new one."""
from __future__ import annotations

import numpy as np

BLOCK = 32
# codes 0..126: multiples of 2^-9 up to 2^-6, then eight to a binade
VALUES = np.array([c * 2.0 ** -9 if c < 8 else (8 + c % 8) / 8 * 2.0 ** (c // 8 - 7) for c in range(127)])
MIDS = (VALUES[1:] + VALUES[:-1]) / 2


def least(top):
    """The smallest e of magnitudes `top`, by trying them from below."""
    e = np.full(np.shape(top), -117)
    for k in range(-117, 119):
        e = np.where(top > 464 * 2.0 ** k, k + 1, e)
    return e


def top(x):
    """Largest finite magnitude of x [..., rows, dh] -> [...]."""
    return np.where(np.isfinite(x), np.abs(x), 0.0).max((-2, -1), initial=0.0)


def encode(x, e):
    """Codes of x with exponents e (which broadcast)."""
    x = np.asarray(x, np.float64)
    fine = np.isfinite(x)
    y = np.abs(np.where(fine, x, 0.0) / 2.0 ** e)
    code = np.searchsorted(MIDS, y, side="left")
    tie = (code < 126) & (y == MIDS[np.minimum(code, 125)])
    code = np.where(tie & (code % 2 == 1), code + 1, code)
    code = code | (np.signbit(np.where(fine, x, 0.0)).astype(int) << 7)
    return np.where(fine, code, 127).astype(np.uint8)


def values(codes, scales):
    """What codes [..., rows, dh] and scales [..., ceil(rows / 32)] stand for."""
    size = np.repeat(2.0 ** (scales.astype(np.float64) - 127), BLOCK, axis=-1)[..., :codes.shape[-2], None]
    mag = np.append(VALUES, np.nan)[codes & 127]
    return np.where(codes & 128, -mag, mag) * size


def append(codes, scales, lens, x):
    """Writes x [B, rows, heads, dh] behind the lens [B] rows of codes [B, heads, capacity, dh] and scales, in place."""
    B, rows, heads, _ = x.shape
    capacity = codes.shape[2]
    for b in range(B):
        first = max(int(lens[b]), 0)
        end = min(int(lens[b]) + rows, capacity)
        for block in range(first // BLOCK, -(-end // BLOCK)):
            start, stop = max(block * BLOCK, first), min((block + 1) * BLOCK, end)
            for h in range(heads):
                new = x[b, start - int(lens[b]):stop - int(lens[b]), h].astype(np.float64)
                e = int(least(top(new)))
                held = slice(block * BLOCK, start)
                if start > block * BLOCK:
                    before = int(scales[b, h, block]) - 127
                    e = max(e, before)
                    codes[b, h, held] = encode(values(codes[b, h, held], np.array([before + 127])), e)
                codes[b, h, start:stop] = encode(new, e)
                scales[b, h, block] = e + 127


def attention(q, k, v, scale, lens, mask=None):
    """q [B,n,H,dh], k and v [B,heads,L,dh] (values), lens [B], mask [B,L] or None -> o [B,n,H,dh], weights [B,heads,L]."""
    B, n, H, dh = q.shape
    heads = k.shape[1]
    group = H // heads
    out, weights = np.zeros(q.shape, np.float64), np.zeros(k.shape[:3])
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
            p /= p.sum(-1, keepdims=True)
            out[b, :, h] = p @ vv
            weights[b, h // group, seen] += p.sum(0)
    return out, weights


def evict(codes, scales, weights, lens, keep, recent, mask=None):
    """-> idx [B,heads,keep] (-1 behind), counts [B], and per (b, h) the codes and scales of the rows kept, as lists of lists."""
    B, heads = codes.shape[:2]
    idx, counts, out = np.full((B, heads, keep), -1, np.int32), np.zeros(B, np.int32), []
    for b in range(B):
        seen = np.arange(codes.shape[2]) < lens[b]
        if mask is not None:
            seen &= mask[b] != 0
        rows = np.flatnonzero(seen)
        counts[b] = min(keep, len(rows))
        late = rows[rows >= lens[b] - recent]
        early = rows[rows < lens[b] - recent]
        out.append([])
        for h in range(heads):
            w = weights[b, h, early].astype(np.float64)
            rank = sorted(range(len(early)), key=lambda i: (not np.isnan(w[i]), 0.0 if np.isnan(w[i]) else -w[i], i))
            stay = np.sort(np.append(early[rank[:counts[b] - len(late)]], late)).astype(int)
            idx[b, h, :counts[b]] = stay
            x = values(codes[b, h], scales[b, h])[stay]
            c, s = np.zeros((len(stay), codes.shape[3]), np.uint8), np.zeros(-(-len(stay) // BLOCK), np.uint8)
            for i in range(len(s)):
                part = slice(i * BLOCK, (i + 1) * BLOCK)
                e = int(least(top(x[part])))
                c[part], s[i] = encode(x[part], e), e + 127
            out[b].append((c, s))
    return idx, counts, out
