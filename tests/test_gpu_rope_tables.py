"""Rotary positions by frequencies of a program's own: whole turns per position do not count, however many.

The angle's fraction of a turn is exact to 2^-50 per position, below 2^-29 at positions up to 2^20; the rest as in test_gpu_rope: 6 * 2^-24 of |x| + |y|."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2512_16483_amd as fv

pytestmark = pytest.mark.gpu

from gpu_util import to_np  # noqa: E402


@pytest.mark.parametrize("size", [0.5, 3.0, 1e4, 1e9, 1e300])
def test_frequencies_of_many_turns(size):
    H, dh, n = 2, 64, 9
    g = np.random.default_rng(3)
    turns = (size * g.uniform(-1, 1, dh // 2)).tolist()
    pos = [0, 1, -1, 7, 12345, 2 ** 20, -2 ** 20, 999983, 2 ** 19 + 1]
    x = g.standard_normal((1, n, H, dh)).astype(np.float32)
    out = torch.empty((1, n, H, dh), device="cuda")
    ctx = fv.Context(hidden=H * dh, heads=H, head_dim=dh, ffn_hidden=64, dtype="f32")
    fv.fvar_rope_apply(ctx, fv.Rope(dim=dh, turns=turns), torch.tensor(pos, dtype=torch.int32, device="cuda").reshape(1, n, 1), 1, n,
                       torch.from_numpy(x).cuda(), q_out=out)
    angle = np.array([[2 * math.pi * float(Fraction(t) * p - round(Fraction(t) * p)) for t in turns] for p in pos])[None, :, None]
    a, b = x[..., :dh // 2].astype(np.float64), x[..., dh // 2:].astype(np.float64)
    want = np.concatenate([a * np.cos(angle) - b * np.sin(angle), a * np.sin(angle) + b * np.cos(angle)], -1)
    room = 6 * 2.0 ** -24 * np.tile(np.abs(a) + np.abs(b), 2)
    assert (np.abs(to_np(out) - want) <= room).all(), float((np.abs(to_np(out) - want) / room).max())
