"""Rotary positions, by their definition, in 64 bits (numpy)."""
from __future__ import annotations

import math

import numpy as np


def frequencies(P, base=10000.0, scaling="none", factor=1.0, original=0.0, low=1.0, high=32.0):
    """Angle per position of each pair of a part of P elements."""
    out = []
    for i in range(P // 2):
        b = base * factor ** (P / (P - 2)) if scaling == "ntk" else base
        f = math.exp(-2.0 * i / P * math.log(b))
        if scaling == "linear":
            f = f / factor
        if scaling == "yarn":
            g = min(max((original * f / (2 * math.pi) - low) / (high - low), 0.0), 1.0)
            f = f * g + f / factor * (1.0 - g)
        out.append(f)
    return np.array(out)


def rotate(x, pos, f, dim, axes=1, interleaved=False, magnitude=1.0):
    """x [B, n, heads, dh], pos [B, n, axes], f: angle per position of each pair of a part."""
    x = np.asarray(x, np.float64)
    y, P = x.copy(), dim // axes
    for a in range(axes):
        for i in range(P // 2):
            one, two = (a * P + 2 * i, a * P + 2 * i + 1) if interleaved else (a * P + i, a * P + P // 2 + i)
            angle = (pos[..., a].astype(np.float64) * f[i])[..., None]
            w = magnitude * np.exp(1j * angle)
            z = (x[..., one] + 1j * x[..., two]) * w
            y[..., one], y[..., two] = z.real, z.imag
    return y
