"""Attention over the 4-bit cache, fp32, where some values are next to nothing beside others."""
import math

import pytest
import torch

import paper_2512_16483_amd as fv

pytestmark = pytest.mark.gpu

from kvb_util import reference  # noqa: E402
from test_gpu_kvb import ctx_of  # noqa: E402


def _cache(B, heads, cap, dh, L):
    t = lambda width: torch.zeros((B, heads, cap, width), dtype=torch.uint8, device="cuda")
    return fv.KVQ(t(dh // 2), t(dh // 2), t(dh // 32), t(dh // 32), len=L)


def _attend(ctx, kv, q, k, v, L):
    """-> output over k and v written into the cache, and what they read back as [B, heads, L, dh]."""
    B, n = q.shape[:2]
    fv.fvar_kvq_append(ctx, fv.KVQ(kv.k, kv.v, kv.k_scale, kv.v_scale), k, v, B, L)
    held = [torch.empty_like(k), torch.empty_like(v)]
    fv.fvar_kvq_read(ctx, kv, B, 0, L, *held)
    o, ws = torch.empty_like(q), torch.empty(fv.fvar_kvq_attention_workspace_bytes(ctx, kv, B, n), dtype=torch.uint8, device="cuda")
    fv.fvar_kvq_attention(ctx, q, kv, B, n, o, ws)
    return o.double(), [x.swapaxes(1, 2).contiguous() for x in held]


@pytest.mark.parametrize("n", [1, 20, 150])
@pytest.mark.parametrize("at", [0, 2, 4])
@pytest.mark.parametrize("less", [60, 150, 200, 215])
def test_fp32_values_far_below_those_of_rows_without_weight(n, at, less):
    """Rows whose values are 2^less times larger than all others, and whose keys get no weight at all: the others count down to 2^-180 of them as
    they are, and from there on no more than they are."""
    H, heads, dh, B, L = 2, 1, 64, 2, 160
    ctx, kv = ctx_of(H, dh, "f32"), _cache(B, heads, L, dh, L)
    g = torch.Generator(device="cuda").manual_seed(less + at)
    draw = lambda *s: torch.randn(s, generator=g, device="cuda")
    q, k, v = draw(B, n, H, dh), draw(B, L, heads, dh), draw(B, L, heads, dh) * 2.0 ** (110 - less)
    far = slice(32 * at, 32 * at + 32)
    q[..., 0], k[..., 0] = 40, 0
    k[:, far, :, 0] = -40                                     # 200 less than the other scores: exp(-150) is 0 in fp32
    v[:, far] = draw(B, 32, heads, dh) * 2.0 ** 110
    o, held = _attend(ctx, kv, q, k, v, L)
    seen = torch.ones((B, L), dtype=torch.bool, device="cuda")
    seen[:, far] = False
    want, _, size, span = reference(q, *held, seen, dh ** -0.5)
    wrong = 2 * dh * 2.0 ** -24 * float(size.max()) + (L + 64) * 2.0 ** -24
    room = span * (wrong if less < 180 else 1 + wrong)
    assert ((o - want).abs() <= room).all(), float(((o - want).abs() / span).max())


@pytest.mark.parametrize("n", [1, 20])
def test_fp32_values_that_are_no_numbers_stay_so_far_below_larger_rows(n):
    H, heads, dh, B, L = 1, 1, 64, 1, 160
    v = torch.randn(B, L, heads, dh, device="cuda") * 2.0 ** -105
    v[:, :32] = 2.0 ** 110
    v[:, 130, :, 9] = math.nan
    o, _ = _attend(ctx_of(H, dh, "f32"), _cache(B, heads, L, dh, L), torch.randn(B, n, H, dh, device="cuda"), torch.randn(B, L, heads, dh, device="cuda"), v, L)
    assert torch.isnan(o[..., :32]).all() and torch.isfinite(o[..., 32:]).all()       # (a scale's 32 elements)
