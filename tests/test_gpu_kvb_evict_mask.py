"""What a program does with a masked cache after an eviction: no row of the cache that received them is hidden, so its mask goes, and the lengths are
those that the call returns."""
import pytest
import torch

import paper_2512_16483_amd as fv

pytestmark = pytest.mark.gpu

from kvb_util import output_room, reference  # noqa: E402
from test_gpu_kvb import attend, ctx_of, empty_cache  # noqa: E402


@pytest.mark.parametrize("here", [True, False])
def test_a_masked_cache_is_cut_down_and_attended_over(here):
    """Of two samples one has fewer rows that are not hidden than are to stay."""
    B, H, dh, L, keep, n = 2, 2, 64, 100, 40, 3
    ctx, g = ctx_of(H, dh, "bf16"), torch.Generator(device="cuda").manual_seed(1)
    draw = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()
    kv = empty_cache(B, H, L, dh)
    fv.fvar_kvb_append(ctx, kv, draw(B, L, H, dh), draw(B, L, H, dh), B, L)
    kv.len = L
    kv.mask = (torch.arange(L, device="cuda") % torch.tensor([[3], [5]], device="cuda") == 0).to(torch.uint8)      # 34 and 20 rows
    kv.mask[0, 50:] = 1
    held = [torch.empty((B, L, H, dh), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    fv.fvar_kvb_read(ctx, kv, B, 0, L, *held)
    to = kv if here else empty_cache(B, H, keep, dh, fill=0x7F)
    q, w = draw(B, n, H, dh), torch.rand((B, H, L), generator=g, device="cuda")
    idx, lens = torch.empty((B, H, keep), dtype=torch.int32, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
    ws = torch.empty(fv.fvar_kvb_evict_workspace_bytes(ctx, kv, B, keep), dtype=torch.uint8, device="cuda")
    fv.fvar_kvb_evict(ctx, kv, w, B, keep, 5, to, w if here else torch.empty((B, H, keep), device="cuda"), lens, idx, ws)
    to.lens, to.mask = lens, None
    assert lens.tolist() == [40, 20]
    k, v = torch.empty((2, B, keep, H, dh), dtype=torch.bfloat16, device="cuda")
    fv.fvar_kvb_read(ctx, to, B, 0, keep, k, v)
    k, v = (x.swapaxes(1, 2).contiguous() for x in (k, v))
    there = torch.arange(keep, device="cuda") < lens[:, None]
    for got, x in ((k, held[0]), (v, held[1])):               # the rows that it says, rounded once more: below 8 by a quarter at most
        want = x.swapaxes(1, 2).gather(2, idx.clamp_min(0).long()[..., None].expand(B, H, keep, dh))
        assert ((got - want).abs()[there[:, None].expand(B, H, keep)] <= 0.25).all()
    want, _, size, span = reference(q, k, v, there, dh ** -0.5)
    room = output_room(want, span, size, float(v.abs().max()), keep, dh, 16)
    assert ((attend(ctx, q, to, "bf16", B, n).double() - want).abs() <= room).all()
