"""Attention over the 8-bit cache where queries, keys and values are no numbers, or among the largest and smallest that their type has."""
import math

import numpy as np
import pytest
import torch

import paper_2512_16483_amd as fv

pytestmark = pytest.mark.gpu

from gpu_util import to_dev  # noqa: E402
from kvb_util import output_room, reference, weight_room  # noqa: E402
from test_gpu_kvb import attend, ctx_of, empty_cache, load, rows_of  # noqa: E402
from test_kvb_host import ways  # noqa: E402

# rows of queries R = n H / heads by their remainder of 64, whole sets of 32 and not; keys by one and by four wavefronts; rows in two shares
ROWS = [(64, 2, 2, 1, 1, 200), (128, 4, 1, 2, 3, 90), (64, 2, 2, 1, 17, 200), (128, 4, 2, 1, 16, 200), (64, 2, 2, 2, 33, 200), (128, 2, 2, 1, 63, 130),
        (64, 1, 1, 1, 65, 300), (128, 2, 1, 2, 48, 100), (64, 4, 4, 1, 200, 333), (64, 2, 1, 1, 130, 300), (64, 16, 16, 16, 20, 60),
        (128, 16, 16, 17, 20, 60), (64, 32, 16, 16, 36, 64), (128, 16, 8, 4, 270, 300)]


def _setup(dtype, dh, H, heads, B, n, L):
    ctx, kv = ctx_of(H, dh, dtype), empty_cache(B, heads, L + 3, dh, fill=0x7F, len=L)
    k, v = (torch.from_numpy(x).cuda() for x in load(kv, rows_of(1, B, L, heads, dh, dtype), rows_of(2, B, L, heads, dh, dtype)))
    return ctx, kv, k, v, to_dev(rows_of(3, B, n, H, dh, dtype, spread=0.2), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dh,H,heads,B,n,L", ROWS)
def test_a_last_query_that_is_no_number_adds_no_weight(dtype, bad, dh, H, heads, B, n, L):
    ctx, kv, k, v, q = _setup(dtype, dh, H, heads, B, n, L)
    clean = attend(ctx, q, kv, dtype, B, n)
    counts = torch.ones((B, n, H), dtype=torch.bool, device="cuda")
    for b in range(0, B, 2):                                  # the last row of the first kv head and of the last
        for h in {H // heads - 1, H - 1}:
            q[b, n - 1, h, 5 + h] = bad
            counts[b, n - 1, h] = False
    w = torch.full((B, heads, L + 3), 0.5, device="cuda")
    o = attend(ctx, q, kv, dtype, B, n, weights=w, add=True)
    assert torch.equal(o[counts], clean[counts])
    assert torch.isnan(o[~counts]).any(-1).all()
    seen = torch.ones((B, L), dtype=torch.bool, device="cuda")
    q[~counts] = 0
    _, want, size, _ = reference(q, k[:, :, :L], v[:, :, :L], seen, dh ** -0.5, counts)
    block = ways(dtype, B, n, H, heads, dh, L, 0)[0]
    off = (w[:, :, :L].double() - 0.5 - want).abs()
    assert (off <= weight_room(want, float(size.max()), dh, block) + 2.0 ** -24 * (0.5 + want)).all(), float(off.max())
    assert (w[:, :, L:] == 0.5).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh,H,heads,B,n,L", ROWS)
def test_a_visible_key_that_is_no_number_leaves_its_head_without_weights(dtype, dh, H, heads, B, n, L):
    ctx, kv, _, _, q = _setup(dtype, dh, H, heads, B, n, L)
    clean = torch.full((B, heads, L + 3), 0.5, device="cuda")
    want = attend(ctx, q, kv, dtype, B, n, weights=clean, add=True)
    kv.k[B - 1, heads - 1, L // 2, 7] = 0x7F
    w = torch.full((B, heads, L + 3), 0.5, device="cuda")
    o = attend(ctx, q, kv, dtype, B, n, weights=w, add=True)
    G = H // heads
    assert torch.isnan(o[B - 1, :, H - G:]).all() and (w[B - 1, heads - 1] == 0.5).all()
    o[B - 1, :, H - G:], w[B - 1, heads - 1] = want[B - 1, :, H - G:], clean[B - 1, heads - 1]
    assert torch.equal(o, want) and torch.equal(w, clean)
    kv.mask = torch.ones((B, L + 3), dtype=torch.uint8, device="cuda")
    kv.mask[B - 1, L // 2] = 0                                # hidden, it has no influence
    attend(ctx, q, kv, dtype, B, n, weights=w)
    assert torch.isfinite(w[:, :, :L]).all() and not w[B - 1, :, L // 2].any()
    assert (w[:, :, :L].sum(-1) - n * G).abs().max() <= 1e-3 * n * G


# blocks of 16 rows, of 128 by four wavefronts and by eight, and in shares
SIZES = [(64, 2, 2, 1, 1, 100), (128, 4, 2, 2, 20, 90), (64, 30, 15, 17, 65, 300), (128, 8, 8, 17, 150, 300), (64, 8, 4, 17, 65, 1100),
         (128, 4, 2, 3, 129, 4100)]


@pytest.mark.parametrize("dh,H,heads,B,n,L", SIZES)
def test_queries_up_to_the_largest_number_of_their_type(dh, H, heads, B, n, L):
    """Elements of 200 to 255 times 2^120, bf16's largest among them, over keys so small that scores are as usual."""
    ctx, kv = ctx_of(H, dh, "bf16"), empty_cache(B, heads, L, dh, len=L)
    g = torch.Generator(device="cuda").manual_seed(5)
    draw = lambda *s: torch.randn(s, generator=g, device="cuda")
    rows = [(draw(B, L, heads, dh) * by).bfloat16() for by in (2.0 ** -124, 1)]
    fv.fvar_kvb_append(ctx, fv.KVB(kv.k, kv.v, kv.k_scale, kv.v_scale), *rows, B, L)
    held = [torch.empty_like(x) for x in rows]
    fv.fvar_kvb_read(ctx, kv, B, 0, L, *held)
    m = torch.randint(200, 256, (B, n, H, dh), generator=g, device="cuda")
    m[:, :, :, 0] = 255
    q = (m * torch.where(draw(B, n, H, dh) < 0, -1, 1) * 2.0 ** 120).bfloat16()
    assert torch.equal(q.double().abs(), m.double() * 2.0 ** 120)
    w = torch.zeros((B, heads, L), device="cuda")
    o = attend(ctx, q, kv, "bf16", B, n, weights=w).double()
    seen = torch.ones((B, L), dtype=torch.bool, device="cuda")
    k, v = (x.swapaxes(1, 2).contiguous() for x in held)
    want, sums, size, span = reference(q, k, v, seen, dh ** -0.5)
    block = ways("bf16", B, n, H, heads, dh, L, 0)[0]
    room = output_room(want, span, size, float(v.abs().max()), L, dh, block)
    assert ((o - want).abs() <= room).all(), float(((o - want).abs() / room).max())
    assert ((w.double() - sums).abs() <= weight_room(sums, float(size.max()), dh, block)).all()


@pytest.mark.parametrize("n", [1, 20, 150])
@pytest.mark.parametrize("at", [0, 2, 4])
@pytest.mark.parametrize("less", [60, 150, 195, 215])
def test_fp32_values_far_below_those_of_a_block_without_weight(n, at, less):
    """A block of values 2^less times larger than all others, whose keys get no weight at all: the others count down to 2^-180 of it as they are, and
    from there on no more than they are."""
    H, heads, dh, B, L = 2, 1, 64, 2, 160
    ctx, kv = ctx_of(H, dh, "f32"), empty_cache(B, heads, L, dh, len=L)
    g = torch.Generator(device="cuda").manual_seed(less + at)
    draw = lambda *s: torch.randn(s, generator=g, device="cuda")
    q, k, v = draw(B, n, H, dh), draw(B, L, heads, dh), draw(B, L, heads, dh) * 2.0 ** (110 - less)
    far = slice(32 * at, 32 * at + 32)
    q[..., 0], k[..., 0] = 40, 0
    k[:, far, :, 0] = -40                                     # 200 less than the other scores: exp(-150) is 0 in fp32
    v[:, far] = draw(B, 32, heads, dh) * 2.0 ** 110
    fv.fvar_kvb_append(ctx, fv.KVB(kv.k, kv.v, kv.k_scale, kv.v_scale), k, v, B, L)
    held = [torch.empty_like(k), torch.empty_like(v)]
    fv.fvar_kvb_read(ctx, kv, B, 0, L, *held)
    o = attend(ctx, q, kv, "f32", B, n).double()
    seen = torch.ones((B, L), dtype=torch.bool, device="cuda")
    seen[:, far] = False                                      # (their part, exp(-150) 2^215 of the others' at most, would show in 64 bits)
    want, _, size, span = reference(q, *[x.swapaxes(1, 2).contiguous() for x in held], seen, dh ** -0.5)
    wrong = 2 * dh * 2.0 ** -24 * float(size.max()) + (L + 64) * 2.0 ** -24
    room = span * (wrong if less < 180 else 1 + wrong)
    assert ((o - want).abs() <= room).all(), float(((o - want).abs() / span).max())


@pytest.mark.parametrize("n", [1, 20])
def test_fp32_values_that_are_no_numbers_stay_so_far_below_a_larger_block(n):
    H, heads, dh, B, L = 1, 1, 64, 1, 160
    ctx, kv = ctx_of(H, dh, "f32"), empty_cache(B, heads, L, dh, len=L)
    v = torch.randn(B, L, heads, dh, device="cuda") * 2.0 ** -105
    v[:, :32] = 2.0 ** 110
    v[:, 130, :, 9] = math.nan
    k = torch.randn_like(v).clamp(-3, 3)
    fv.fvar_kvb_append(ctx, fv.KVB(kv.k, kv.v, kv.k_scale, kv.v_scale), k, v, B, L)
    o = attend(ctx, torch.randn(B, n, H, dh, device="cuda"), kv, "f32", B, n)
    assert torch.isnan(o[..., 9]).all() and torch.isfinite(o[..., :9]).all() and torch.isfinite(o[..., 10:]).all()
