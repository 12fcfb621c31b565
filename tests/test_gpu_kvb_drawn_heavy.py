"""Attention over the 8-bit cache at drawn sizes, over queries, keys and values with heavy tails: rows, elements, channels and blocks of very different sizes.
Against the same in 64 bits, within what the kernels' number formats leave (kvb_util)."""
import random

import pytest
import torch

import paper_2512_16483_amd as fv

pytestmark = pytest.mark.gpu

from gpu_util import tdtype  # noqa: E402
from kvb_util import bounds, output_room, reference, weight_room  # noqa: E402
from test_gpu_kvb import attend, ctx_of, empty_cache  # noqa: E402
from test_kvb_host import ways  # noqa: E402


def _draw(rng):
    while True:
        c = dict(dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), dh=rng.choice([64, 128]), H=rng.choice([1, 2, 4, 6, 8, 16, 30, 32]),
                 B=rng.choice([1, 2, 3, 5, 8, 17, 33]), n=rng.choice([1, 2, 5, 17, 20, 33, 64, 65, 100, 129, 200, 300, 700]),
                 L=rng.choice([1, 2, 33, 65, 127, 200, 400, 777, 1500, 3000, 5000]), tails=rng.choice(["rows", "elements", "channels", "blocks", "all"]),
                 masked=rng.random() < 0.4)
        c["heads"] = rng.choice([h for h in range(1, c["H"] + 1) if c["H"] % h == 0])
        if c["B"] * c["n"] * c["H"] * c["L"] <= 3e7:
            return c


@pytest.mark.parametrize("seed", range(4))
def test_drawn_calls_over_heavy_tails(seed):
    rng, g = random.Random(seed), torch.Generator(device="cuda").manual_seed(seed)
    draw = lambda *s: torch.randn(s, generator=g, device="cuda")
    for _ in range(150):
        c = _draw(rng)
        B, n, L, H, heads, dh, dtype, tails = (c[x] for x in ("B", "n", "L", "H", "heads", "dh", "dtype", "tails"))
        block = ways(dtype, B, n, H, heads, dh, L, 0)[0]
        print(f"[kvb heavy] {c} by {block}", end=" ", flush=True)
        q, k, v = draw(B, n, H, dh), draw(B, L, heads, dh), draw(B, L, heads, dh)
        if tails in ("rows", "all"):
            q, k, v = q * torch.exp(0.5 * draw(B, n, H, 1)), k * torch.exp(draw(B, L, heads, 1)), v * torch.exp(2 * draw(B, L, heads, 1))
        if tails in ("elements", "all"):
            q, k, v = q * torch.exp(0.7 * draw(B, n, H, dh)), k * torch.exp(0.7 * draw(B, L, heads, dh)), v * torch.exp(2 * draw(B, L, heads, dh))
        if tails in ("channels", "all"):
            some, by = rng.sample(range(dh), rng.choice([1, 2, 5])), rng.choice([3, 8, 15])
            q[..., some] *= by
            k[..., some] *= by
        if tails in ("blocks", "all"):
            powers = torch.randint(-30, 30, (B, -(-L // 32), 1, 1), generator=g, device="cuda")
            v = v * torch.exp2(powers.float()).repeat_interleave(32, 1)[:, :L]
        q, k, v = ((x * by).to(tdtype(dtype)) for x, by in ((q, rng.choice([0.3, 1, 1, 2])), (k, 1), (v, 1)))
        ctx, kv = ctx_of(H, dh, dtype), empty_cache(B, heads, L, dh, fill=127)
        fv.fvar_kvb_append(ctx, kv, k, v, B, L)
        kv.len = L
        held = [torch.empty_like(k), torch.empty_like(v)]
        fv.fvar_kvb_read(ctx, kv, B, 0, L, *held)
        k, v = (x.swapaxes(1, 2).contiguous() for x in held)
        seen = torch.ones((B, L), dtype=torch.bool, device="cuda")
        if c["masked"]:
            kv.mask = (torch.rand((B, L), generator=g, device="cuda") < rng.choice([0.05, 0.5, 0.9])).to(torch.uint8)
            seen = kv.mask != 0
        w = torch.zeros((B, heads, L), device="cuda")
        o = attend(ctx, q, kv, dtype, B, n, weights=w).double()
        if block == 128:
            want, room, sums, w_room, _, _ = bounds(q, k, v, kv.k_scale, seen, dh ** -0.5)
        else:
            want, sums, size, span = reference(q, k, v, seen, dh ** -0.5)
            w_room = weight_room(sums, 2 * float(size.max()), dh, 16)          # (in p and in its sum)
            if dtype == "bf16":
                room = output_room(want, span, size, float(v.double().abs().max()), L, dh, 16)
            else:                                             # fp32 throughout: sums of L numbers, exponentials, their least, 2^-126, the result's own rounding
                room = (torch.expm1(2 * dh * 2.0 ** -24 * size * 2)[..., None] + (L + 64) * 2.0 ** -24 + 2.0 ** -20) * span + 2.0 ** -23 * want.abs()
                room = room + L * 2.0 ** -125 * float(v.double().abs().max()) + 1e-38
        share, w_share = float(((o - want).abs() / room).max()), float(((w.double() - sums).abs() / w_room).max())
        print(f"{share:.2g} of the room, weights {w_share:.2g}", flush=True)
        assert share <= 1 and w_share <= 1, (c, share, w_share)
