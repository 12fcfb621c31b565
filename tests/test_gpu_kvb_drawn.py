"""Attention over the 8-bit cache at drawn sizes, types, lengths, masks, distances between queries and sizes of scores and values, after rows were
written into it in two calls and read back: against the same in 64 bits, within the library's bars.  Rows' weights: as in test_gpu_kvb, and where blocks of
128 rows are attended at once, whose scores are added up to 2^-14 of scale sum |q k|, that much more."""
import random

import pytest
import torch

import paper_2512_16483_amd as fv

pytestmark = pytest.mark.gpu

from gpu_util import TOL, tdtype  # noqa: E402
from test_gpu_kvb import NORM, attend, ctx_of, empty_cache  # noqa: E402
from test_kvb_host import ways  # noqa: E402


def _draw(rng):
    while True:
        c = dict(dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), dh=rng.choice([64, 128]), H=rng.choice([1, 2, 4, 6, 8, 16, 30, 32]),
                 B=rng.choice([1, 1, 2, 3, 5, 8, 17]), n=rng.choice([1, 1, 2, 5, 16, 17, 33, 64, 100, 128, 129, 200, 300, 500, 1000]),
                 L=rng.choice([1, 2, 31, 33, 63, 65, 127, 200, 400, 777, 1500, 3000, 5000, 9000]), more=rng.randrange(70),
                 ragged=rng.random() < 0.4, masked=rng.random() < 0.4, apart=rng.random() < 0.5)
        c["heads"] = rng.choice([h for h in range(1, c["H"] + 1) if c["H"] % h == 0])
        if c["B"] * c["n"] * c["H"] * c["L"] <= 1.2e8:
            return c


def _reference(q, k, v, seen, scale):
    """-> output, weights of rows, the largest scale sum |q k|."""
    out, group, most = torch.zeros(q.shape, dtype=torch.float64, device="cuda"), q.shape[2] // k.shape[2], 0.0
    w = torch.zeros((k.shape[0], k.shape[2], k.shape[1]), dtype=torch.float64, device="cuda")
    for b in range(q.shape[0]):
        at = seen[b].nonzero().flatten()
        for h in range(q.shape[2] if len(at) else 0):
            qq, kk, vv = q[b, :, h].double(), k[b, at, h // group].double().T.contiguous(), v[b, at, h // group].double()
            p = torch.softmax(qq @ kk * scale, -1)
            out[b, :, h] = p @ vv
            w[b, h // group, at] += p.sum(0)
            most = max(most, float((qq.abs() @ kk.abs()).max()) * scale)
    return out, w, most


@pytest.mark.parametrize("seed", range(6))
def test_drawn_calls(seed):
    rng, g = random.Random(seed), torch.Generator(device="cuda").manual_seed(seed)
    for _ in range(40):
        c = _draw(rng)
        B, n, L, H, heads, dh, dtype, cap = c["B"], c["n"], c["L"], c["H"], c["heads"], c["dh"], c["dtype"], c["L"] + c["more"]
        way = ways(dtype, B, n, H, heads, dh, cap if c["ragged"] else L, c["ragged"])
        print(f"[kvb drawn] {c} by {way}", end=" ", flush=True)
        spread = rng.choice([0.0, 0.5, 1.0])

        def rows(m, h, s):
            return torch.randn(B, m, h, dh, generator=g, device="cuda") * torch.exp(s * torch.randn(B, m, h, 1, generator=g, device="cuda"))

        k, v = rows(L, heads, spread), rows(L, heads, spread) * rng.choice([1, 1e-3, 1e4, 2.0 ** 100, 2.0 ** -100])
        q = rows(n, H, 0.2) * rng.choice([0.3, 1, 1, 2, 3])
        if dtype == "bf16" and rng.random() < 0.4:            # some elements of the queries far larger, the keys' as much smaller
            some, by = rng.sample(range(dh), rng.choice([1, 2, 8])), rng.choice([20, 100, 1000])
            q[..., some] *= by
            k[..., some] /= by
        q, k, v = (x.to(tdtype(dtype)) for x in (q, k, v))
        lens = torch.tensor([rng.randrange(L + 1) for _ in range(B)], dtype=torch.int32, device="cuda") if c["ragged"] else None
        mask = None
        if c["masked"]:
            mask = (torch.rand(B, cap, generator=g, device="cuda") < rng.choice([0.02, 0.5, 0.9])).to(torch.uint8)
            mask[rng.randrange(B)] *= rng.random() < 0.7
        ctx, kv = ctx_of(H, dh, dtype), empty_cache(B, heads, cap, dh, fill=127)
        first = rng.randrange(L)
        if first:
            fv.fvar_kvb_append(ctx, kv, k[:, :first].contiguous(), v[:, :first].contiguous(), B, first)
            kv.len = first
        fv.fvar_kvb_append(ctx, kv, k[:, first:].contiguous(), v[:, first:].contiguous(), B, L - first)
        kv.len, kv.lens, kv.mask = L, lens, mask
        held = [torch.empty_like(k), torch.empty_like(v)]
        fv.fvar_kvb_read(ctx, fv.KVB(kv.k, kv.v, kv.k_scale, kv.v_scale, len=L), B, 0, L, *held)
        if c["apart"]:
            q = torch.empty(B, n, H * dh + 64, dtype=q.dtype, device="cuda").narrow(2, 0, H * dh).copy_(q.reshape(B, n, H * dh))
        w = torch.full((B, heads, cap), 7.0, device="cuda")
        o = attend(ctx, q, kv, dtype, B, n, weights=w).double()
        assert torch.equal(attend(ctx, q, kv, dtype, B, n).double(), o)
        there = (torch.arange(L, device="cuda") < (lens[:, None] if lens is not None else L)).expand(B, L)
        seen = there & (mask[:, :L] != 0) if mask is not None else there
        want, sums, most = _reference(q.reshape(B, n, H, dh), *held, seen, dh ** -0.5)
        room = 2 * dh * 2.0 ** -24 * most + 2.0 ** -20 + 2.0 ** -18 + (2.0 ** -14 * most if way[0] == 128 else 0)
        off = torch.where(there[:, None], (w[:, :, :L] - sums).abs() - room * sums, (w[:, :, :L] - 7).abs())
        size = want.abs().max().clamp_min(1e-300)
        err, want = (o - want) / size, want / size
        norm = float(err.norm() / want.norm().clamp_min(1e-300))
        worst = float((err.abs() / want.abs().clamp_min(want.square().mean().sqrt().clamp_min(1e-300))).max())
        print(f"norm {norm:.2g} max {worst:.2g} weights {float(off.max()):.2g}", flush=True)
        assert norm <= NORM[dtype] and worst <= TOL[dtype] and float(off.max()) <= 1e-30, (c, norm, worst)
        assert (w[:, :, L:] == 7).all()
