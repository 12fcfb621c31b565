"""Attention over the 4-bit cache at drawn sizes, types, lengths, masks, distances between queries and sizes of scores and values, after rows were
quantised into it and read back: against the same in 64 bits, within the library's bars."""
import random

import pytest
import torch

import paper_2512_16483_amd as fv

pytestmark = pytest.mark.gpu

from gpu_util import TOL, tdtype  # noqa: E402
from test_gpu_kvq import NORM, _attend, _ctx, _empty_cache  # noqa: E402
from test_kvq_host import ways  # noqa: E402


def _draw(rng):
    while True:
        c = dict(dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), dh=rng.choice([64, 128]), H=rng.choice([1, 2, 4, 6, 8, 16, 30, 32]),
                 B=rng.choice([1, 1, 2, 3, 5, 8, 17]), n=rng.choice([1, 1, 2, 5, 16, 33, 64, 100, 128, 129, 200, 300, 500, 1000]),
                 L=rng.choice([1, 2, 31, 33, 63, 65, 127, 200, 400, 777, 1500, 3000, 5000, 9000]), more=rng.randrange(70),
                 ragged=rng.random() < 0.4, masked=rng.random() < 0.4, apart=rng.random() < 0.5)
        c["heads"] = rng.choice([h for h in range(1, c["H"] + 1) if c["H"] % h == 0])
        if c["B"] * c["n"] * c["H"] * c["L"] <= 1.2e8:
            return c


def _reference(q, k, v, seen, scale):
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    group = q.shape[2] // k.shape[2]
    for b in range(q.shape[0]):
        at = seen[b].nonzero().flatten()
        for h in range(q.shape[2] if len(at) else 0):
            kk, vv = k[b, at, h // group].double(), v[b, at, h // group].double()
            out[b, :, h] = torch.softmax(q[b, :, h].double() @ kk.T.contiguous() * scale, -1) @ vv
    return out


@pytest.mark.parametrize("seed", range(6))
def test_drawn_calls(seed):
    rng, g = random.Random(seed), torch.Generator(device="cuda").manual_seed(seed)
    worst = {}
    for _ in range(40):
        c = _draw(rng)
        B, n, L, H, heads, dh, dtype, cap = c["B"], c["n"], c["L"], c["H"], c["heads"], c["dh"], c["dtype"], c["L"] + c["more"]
        print(f"[kvq drawn] {c} by {ways(dtype, B, n, H, heads, dh, cap if c['ragged'] else L, c['ragged'])}", end=" ", flush=True)
        spread = rng.choice([0.0, 0.5, 1.0])

        def rows(m, h, s):
            return torch.randn(B, m, h, dh, generator=g, device="cuda") * torch.exp(s * torch.randn(B, m, h, 1, generator=g, device="cuda"))

        k, v = rows(L, heads, spread), rows(L, heads, spread) * rng.choice([1, 1e-3, 1e4, 2.0 ** 100, 2.0 ** -100])
        q = rows(n, H, 0.2) * rng.choice([0.3, 1, 1, 2] + ([4, 8, 16] if dtype == "bf16" else []))
        if dtype == "bf16" and rng.random() < 0.4:            # some elements of the queries far larger, the keys' as much smaller
            some, by = rng.sample(range(dh), rng.choice([1, 2, 8])), rng.choice([20, 100, 1000, 1e5])
            q[..., some] *= by
            k[..., some] /= by
        q, k, v = (x.to(tdtype(dtype)) for x in (q, k, v))
        lens = torch.tensor([rng.randrange(L + 1) for _ in range(B)], dtype=torch.int32, device="cuda") if c["ragged"] else None
        mask = None
        if c["masked"]:
            mask = (torch.rand(B, cap, generator=g, device="cuda") < rng.choice([0.02, 0.5, 0.9])).to(torch.uint8)
            mask[rng.randrange(B)] *= rng.random() < 0.7
        ctx, kv = _ctx(H, dh, dtype), _empty_cache(B, heads, cap, dh, fill=255)
        fv.fvar_kvq_append(ctx, kv, k, v, B, L)
        kv.len, kv.lens, kv.mask = L, lens, mask
        held = [torch.empty_like(k), torch.empty_like(v)]
        fv.fvar_kvq_read(ctx, fv.KVQ(kv.k, kv.v, kv.k_scale, kv.v_scale, len=L), B, 0, L, *held)
        if c["apart"]:
            q = torch.empty(B, n, H * dh + 64, dtype=q.dtype, device="cuda").narrow(2, 0, H * dh).copy_(q.reshape(B, n, H * dh))
        o = _attend(ctx, q, kv, dtype, B, n).double()
        seen = torch.arange(L, device="cuda") < (lens[:, None] if lens is not None else L)
        seen = (seen & (mask[:, :L] != 0) if mask is not None else seen).expand(B, L)
        want = _reference(q.reshape(B, n, H, dh), *held, seen, dh ** -0.5)
        size = want.abs().max().clamp_min(1e-300)
        err, want = (o - want) / size, want / size
        norm = float(err.norm() / want.norm().clamp_min(1e-300))
        most = float((err.abs() / want.abs().clamp_min(want.square().mean().sqrt().clamp_min(1e-300))).max())
        print(f"norm {norm:.2g} max {most:.2g}", flush=True)
        assert norm <= NORM[dtype] and most <= TOL[dtype], (c, norm, most)
        worst[dtype] = max(worst.get(dtype, (0, 0)), (most, norm))
    print(f"[kvq drawn] seed {seed}: most {worst}", flush=True)
