"""Attention over the 8-bit cache by blocks of 128 rows (kvb_attn_tiles_kernel), in each of the ways in which they are run, over scores and values of
every size, what is no number, and masks that leave little: against the same in 64 bits.  Each size says how it is run, and is held to that."""
import math

import numpy as np
import pytest
import torch

import paper_2512_16483_amd as fv
import workloads as wl

pytestmark = pytest.mark.gpu

from gpu_util import to_dev  # noqa: E402
from kvb_util import bounds, reference  # noqa: E402
from test_gpu_kvb import attend, check, ctx_of, empty_cache, fill, rows_of  # noqa: E402
from test_kvb_host import ways  # noqa: E402

# head_dim, heads, kv heads, samples, queries, rows held; the way: wavefronts, shares.  64-wide rows by four wavefronts, two and three of them per SIMD, whole and
# in shares; by eight, which are two groups with half of the keys each; 128-wide ones by four and by eight
WAYS = [(64, 30, 15, 17, 65, 300, 4, 1), (64, 2, 1, 33, 65, 4100, 4, 7), (64, 30, 15, 64, 65, 100, 4, 1), (64, 30, 30, 64, 17, 700, 4, 2), (64, 8, 4, 17, 65, 1100, 8, 1),
        (64, 16, 16, 2, 65, 4100, 8, 8), (128, 8, 8, 17, 150, 300, 4, 1), (128, 2, 1, 33, 65, 4100, 4, 7), (128, 16, 8, 8, 65, 700, 8, 1), (128, 4, 2, 3, 129, 4100, 8, 8)]
every_way = pytest.mark.parametrize("dh,H,heads,B,n,L,waves,shares", WAYS)
H_NAN = 0x7F


def _held(dh, H, heads, B, n, L, waves, shares, k, v):
    """A cache over k and v [B, L, heads, dh], and what it holds as [B, heads, L, dh]."""
    assert ways("bf16", B, n, H, heads, dh, L, 0) == (128, waves, shares)
    ctx, kv = ctx_of(H, dh, "bf16"), empty_cache(B, heads, L, dh, fill=H_NAN)
    fv.fvar_kvb_append(ctx, kv, k.bfloat16(), v.bfloat16(), B, L)
    kv.len = L
    held = [torch.empty((B, L, heads, dh), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    fv.fvar_kvb_read(ctx, kv, B, 0, L, *held)
    return ctx, kv, *(x.swapaxes(1, 2).contiguous() for x in held)


def _draws(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *s: torch.randn(s, generator=g, device="cuda")


def _look(tag, ctx, kv, q, k, v, seen):
    """Output and weights of a call against the reference, within what the kernels' number formats leave."""
    B, n, H, dh = q.shape
    heads, L = k.shape[1], k.shape[2]
    w = torch.full((B, heads, L), 0.25, device="cuda")
    o = attend(ctx, q, kv, "bf16", B, n, weights=w, add=True).double()
    want, room, sums, weight_room, size, taken = bounds(q, k, v, kv.k_scale, seen, dh ** -0.5)
    share = float(((o - want).abs() / room).max())
    w_share = float(((w.double() - 0.25 - sums).abs() / (weight_room + 2.0 ** -24 * (0.25 + sums))).max())
    norm = float((o - want).norm() / want.norm().clamp_min(1e-300))
    print(f"[kvb blocks] {tag}: {share:.3g} of the room, norm {norm:.3g}, scores' sizes to {float(size):.3g}, weights {w_share:.3g} of theirs, {taken:.3g} as "
          "they are", flush=True)
    assert share <= 1 and w_share <= 1


def _all_seen(B, L):
    return torch.ones((B, L), dtype=torch.bool, device="cuda")


@every_way
@pytest.mark.parametrize("size", [1e-3, 1.0, 30.0])
def test_scores_of_every_size(dh, H, heads, B, n, L, waves, shares, size):
    """Up to hundreds; keys grow along the cache, so that references are left again and again."""
    draw = _draws(1)
    rise = torch.linspace(0.2, 1.5, L, device="cuda")[:, None, None]
    q = (draw(B, n, H, dh) * size).bfloat16()
    ctx, kv, k, v = _held(dh, H, heads, B, n, L, waves, shares, draw(B, L, heads, dh) * rise, draw(B, L, heads, dh))
    _look(f"scores {size}", ctx, kv, q, k, v, _all_seen(B, L))


@every_way
@pytest.mark.parametrize("by", [2.0, 6.0, 20.0])
@pytest.mark.parametrize("some", ["all queries", "a few queries", "a few keys"])
def test_a_channel_far_larger_than_the_others(dh, H, heads, B, n, L, waves, shares, by, some):
    """One element of queries and keys `by` times the others' size, its products up to hundreds: the others count beside it."""
    draw = _draws(9)
    q, k = draw(B, n, H, dh), draw(B, L, heads, dh)
    at = dh // 3
    q[..., at] = by * (1 + 0.02 * draw(B, n, H)) if some != "a few queries" else torch.where(draw(B, n, 1) < 1.5, q[..., at], by)
    k[..., at] = by * (1 + 0.02 * draw(B, L, heads)) if some != "a few keys" else torch.where(draw(B, L, 1) < 2, k[..., at], by)
    ctx, kv, k, v = _held(dh, H, heads, B, n, L, waves, shares, k, draw(B, L, heads, dh))
    _look(f"channel x {by} of {some}", ctx, kv, q.bfloat16(), k, v, _all_seen(B, L))


@every_way
def test_scores_beyond_all_exponentials(dh, H, heads, B, n, L, waves, shares):
    """Scores of 10^11: where the best one stands out by more than all errors, the output is its value."""
    draw = _draws(2)
    q = (draw(B, n, H, dh) * 1e10).bfloat16()
    ctx, kv, k, v = _held(dh, H, heads, B, n, L, waves, shares, draw(B, L, heads, dh), draw(B, L, heads, dh))
    w = torch.zeros((B, heads, L), device="cuda")
    o = attend(ctx, q, kv, "bf16", B, n, weights=w)
    assert torch.isfinite(o).all() and torch.isfinite(w).all() and (w >= 0).all() and (w <= n * H // heads * 1.0001).all()
    want, _, size, _ = reference(q, k, v, _all_seen(B, L), dh ** -0.5)
    clear, G = 0, H // heads
    for b in range(0, B, max(1, B // 3)):
        for h in range(H):
            s = q[b, :, h].double() @ k[b, h // G].double().T.contiguous() * dh ** -0.5
            two = torch.topk(s, 2, -1).values
            alone = two[:, 0] - two[:, 1] > 60 + 2 * 2.0 ** -14 * size[b, :, h]
            clear += int(alone.sum())
            assert ((o[b, :, h].double() - want[b, :, h]).abs() <= 2.0 ** -8 * want[b, :, h].abs() + 1e-30)[alone].all()
    assert clear > 0


@every_way
@pytest.mark.parametrize("e", [-40, -17, -9, 9, 17, 40, 100])
@pytest.mark.parametrize("weigh", [True, False])
def test_blocks_of_values_of_every_size(dh, H, heads, B, n, L, waves, shares, e, weigh):
    """Three blocks of 32 rows, first, within and last, with values 2^e of the others' sizes; with a weight like theirs, or with none, so that
    what is left has to come out at its own size beside them."""
    draw = _draws(3 + e)
    q, k, v = draw(B, n, H, dh) * 0.7, draw(B, L, heads, dh), draw(B, L, heads, dh)
    last = (L - 1) // 32
    far = torch.isin(torch.arange(L, device="cuda") // 32, torch.tensor([0, last // 2, last], device="cuda"))
    v[:, far] *= 2.0 ** e
    if not weigh:
        q[..., 0], k[..., 0] = 48, -48 * far[:, None].float()                      # 200 and more below the other scores
    ctx, kv, k, v = _held(dh, H, heads, B, n, L, waves, shares, k, v)
    _look(f"values 2^{e}", ctx, kv, q.bfloat16(), k, v, _all_seen(B, L))


@every_way
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_queries_that_are_no_numbers(dh, H, heads, B, n, L, waves, shares, bad):
    draw = _draws(4)
    q = draw(B, n, H, dh).bfloat16()
    ctx, kv, k, v = _held(dh, H, heads, B, n, L, waves, shares, draw(B, L, heads, dh), draw(B, L, heads, dh))
    clean = attend(ctx, q, kv, "bf16", B, n)
    counts = torch.ones((B, n, H), dtype=torch.bool, device="cuda")
    for b, i, h in ((0, 0, 0), (0, n - 1, H - 1), (B - 1, n // 2, 0), (B - 1, n - 1, H // heads - 1)):
        q[b, i, h, 7] = bad
        counts[b, i, h] = False
    w = torch.zeros((B, heads, L), device="cuda")
    o = attend(ctx, q, kv, "bf16", B, n, weights=w)
    assert torch.isnan(o[~counts]).all() and torch.equal(o[counts], clean[counts])
    q[~counts] = 0
    _, _, want, room, _, _ = bounds(q, k, v, kv.k_scale, _all_seen(B, L), dh ** -0.5, counts)
    assert ((w.double() - want).abs() <= room).all()


@every_way
def test_keys_and_values_that_are_no_numbers(dh, H, heads, B, n, L, waves, shares):
    """A key: all rows that see it, and their weights are none.  A value: its element of all rows.  Hidden, neither shows."""
    draw, G = _draws(5), H // heads
    q = draw(B, n, H, dh).bfloat16()
    ctx, kv, k, v = _held(dh, H, heads, B, n, L, waves, shares, draw(B, L, heads, dh), draw(B, L, heads, dh))
    clean = torch.zeros((B, heads, L), device="cuda")
    want = attend(ctx, q, kv, "bf16", B, n, weights=clean)
    for at in (0, L // 2 + 5, L - 1):
        codes = kv.k.clone(), kv.v.clone()
        kv.k[0, heads - 1, at, 3] = kv.v[B - 1, 0, at, dh - 1] = H_NAN
        w = torch.zeros_like(clean)
        o = attend(ctx, q, kv, "bf16", B, n, weights=w)
        assert torch.isnan(o[0, :, H - G:]).all() and not w[0, heads - 1].any() and torch.isnan(o[B - 1, :, :G, dh - 1]).all()
        o[0, :, H - G:], o[B - 1, :, :G, dh - 1], w[0, heads - 1] = want[0, :, H - G:], want[B - 1, :, :G, dh - 1], clean[0, heads - 1]
        assert torch.equal(o, want) and torch.equal(w, clean)
        kv.mask = torch.ones((B, L), dtype=torch.uint8, device="cuda")
        kv.mask[:, at] = 0
        _look(f"hidden {at}", ctx, kv, q, k, v, kv.mask != 0)
        kv.mask = None
        kv.k.copy_(codes[0])
        kv.v.copy_(codes[1])


@every_way
@pytest.mark.parametrize("kind", ["one row", "a row in every share", "second half of a tile", "first rows", "last rows", "one sample", "lengths"])
def test_masks_that_leave_little(dh, H, heads, B, n, L, waves, shares, kind):
    """Groups, shares and halves of tiles in which nothing is seen, whatever hidden rows hold."""
    draw = _draws(6)
    q = draw(B, n, H, dh).bfloat16()
    ctx, kv, k, v = _held(dh, H, heads, B, n, L, waves, shares, draw(B, L, heads, dh), draw(B, L, heads, dh))
    seen = torch.zeros((B, L), dtype=torch.bool, device="cuda")
    rows = torch.arange(L, device="cuda")
    if kind == "one row":
        seen[torch.arange(B), torch.arange(B) * 997 % L] = True
    elif kind == "a row in every share":
        seen[:, 13::max(1, L // 16)] = True
    elif kind == "second half of a tile":
        seen |= (rows // 32 % 2 == 1) & (rows % 3 == 0)
    elif kind == "first rows":
        seen[:, :5] = True
    elif kind == "last rows":
        seen[:, -5:] = True
    elif kind == "one sample":
        seen[B // 2] = True
    lens = None
    if kind == "lengths":
        lens = torch.tensor([(b * 37) % (L + 1) if b % 5 else (0, 1, 33, 64, L)[b // 5 % 5] for b in range(B)], dtype=torch.int32, device="cuda")
        seen = rows < lens[:, None]
        kv.lens = lens
    else:
        kv.mask = seen.to(torch.uint8) * 2
    hidden = ~seen[:, None, :, None].expand(B, heads, L, 1)
    kv.k.masked_fill_(hidden, H_NAN)
    kv.v.masked_fill_(hidden, 0xFF)
    w = torch.full((B, heads, L), 9.0, device="cuda")
    want, room, sums, weight_room, _, _ = bounds(q, k, v, kv.k_scale, seen, dh ** -0.5)
    o = attend(ctx, q, kv, "bf16", B, n, weights=w).double()
    assert ((o - want).abs() <= room).all() and not o[~seen.any(-1)].any()
    there = (rows < lens[:, None] if lens is not None else torch.ones_like(seen))[:, None].expand(B, heads, L)
    assert ((w.double() - sums).abs() <= weight_room)[there].all() and (w[~there] == 9).all()


@pytest.mark.parametrize("d,H,B,M,keep,Lp,waves,shares", [(512, 8, 4, 320, 300, 800, 8, 2), (1024, 8, 3, 250, 250, 850, 8, 2), (2048, 16, 17, 140, 129, 171, 4, 1)])
@pytest.mark.parametrize("turned", [False, True])
def test_block_over_the_cache_by_blocks_of_128_rows(d, H, B, M, keep, Lp, waves, shares, turned):
    """The block call against the calls that it is made of: the same cache and the same weights, bit for bit, and x + attention where W_o = 1 and the MLP is
    0."""
    dh, F, cap = d // H, 64, Lp + keep
    assert ways("bf16", B, keep, H, H, dh, cap, 0) == (128, waves, shares)
    g = np.random.default_rng(7)
    x = to_dev(wl.activations_lowrank(B, M, d, seed=8, bf16=True), "bf16")
    w = {"w_qkv": 0.05 * g.standard_normal((3 * d, d)), "b_qkv": 0.1 * g.standard_normal(3 * d), "w_o": np.eye(d), "w_fc1": np.zeros((F, d)),
         "w_fc2": np.zeros((d, F))}
    w = {name: to_dev(wl.round_to_bf16(a.astype(np.float32)), "bf16") for name, a in w.items()}
    rolled = dict(w, w_qkv=w["w_qkv"].roll(d, 0).contiguous(), b_qkv=w["b_qkv"].roll(d, 0).contiguous())       # q rows come out as K rows
    ctx = fv.Context(hidden=d, heads=H, head_dim=dh, ffn_hidden=F, dtype="bf16")
    idx = np.stack([np.sort(g.permutation(M)[:keep]) for _ in range(B)]).astype(np.int32)
    idx_d = torch.from_numpy(idx).cuda()
    bf16 = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")

    def plain(weights):
        K, V, y = bf16(B, keep, H, dh), bf16(B, keep, H, dh), bf16(B, keep, d)
        ws = torch.empty(fv.fvar_block_workspace_bytes(ctx, B, keep), dtype=torch.uint8, device="cuda")
        fv.fvar_block_forward_pruned(ctx, weights, x, B, M, idx_d, keep, K, V, keep, 0, y, ws)
        return K, V

    (kn, vn), (qn, _) = plain(w), plain(rolled)
    r = fv.Rope(dim=32, axes=2) if turned else None
    pos = torch.from_numpy(np.stack([idx // 16, idx % 16], -1).astype(np.int32)).cuda() if turned else None
    if turned:
        fv.fvar_rope_apply(ctx, r, pos, B, keep, qn, kn)
    one, two = (empty_cache(B, H, cap, dh, fill=H_NAN) for _ in range(2))
    for kv in (one, two):
        fill(kv, Lp)
        kv.len = Lp
    fv.fvar_kvb_append(ctx, one, kn, vn, B, keep)
    one.len = cap
    sums, got = torch.full((B, H, cap), 0.5, device="cuda"), torch.full((B, H, cap), 0.5, device="cuda")
    att = attend(ctx, qn, one, "bf16", B, keep, weights=sums, add=True)
    ws = torch.full((fv.fvar_block_kvb_workspace_bytes(ctx, two, B, keep, weights=True),), 255, dtype=torch.uint8, device="cuda")
    y = bf16(B, keep, d)
    if keep == M:
        fv.fvar_block_forward_dense_kvb(ctx, w, x, B, M, two, y, ws, rope=r, pos=pos, weights=got, add=True)
    else:
        fv.fvar_block_forward_pruned_kvb(ctx, w, x, B, M, idx_d, keep, two, y, ws, rope=r, pos=pos, weights=got, add=True)
    for name in ("k", "v", "k_scale", "v_scale"):
        assert torch.equal(getattr(one, name), getattr(two, name))
    assert torch.equal(sums, got)
    xk = torch.stack([x[b, idx_d[b].long()] for b in range(B)])
    check(f"block {B}x{keep}", y, (xk.double() + att.reshape(B, keep, d).double()).cpu().numpy(), "bf16")
