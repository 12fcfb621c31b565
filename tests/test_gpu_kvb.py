"""The 8-bit cache on the GPU through the C ABI, against its definition in 64 bits.

Writing and reading back are exact: codes and scales have to be the oracle's bit for bit.  Attention in bf16: the output is rounded
once (2^-8 relative at most, 1.7e-3 rms), the weights on the way to 11 bits (2.9e-4 rms, each independently): 2-norm of the error at most
3e-3 of the result's.  In fp32 sums of a few thousand terms leave at most 5e-6.  The largest error of one element is held to the library's bars (2e-2,
1e-4 of max(|o|, rms)).
The weights of rows are sums of p = exp(s - m) / l in fp32: a score of D products, whose order is free, is off by at most D 2^-24 of sum |q k|, here twice (in
l and in p), exp and the division by 2^-22: relative to the weight at most 2 D 2^-24 scale max sum |q k| + 2^-20, sums of positive numbers add at
most their number of steps times 2^-24, below 2^-18 for what is tested."""
import math

import numpy as np
import pytest
import torch

import paper_2512_16483_amd as fv
import workloads as wl
from oracle import kvb

pytestmark = pytest.mark.gpu

from gpu_util import TOL, rel_err, tdtype, to_dev, to_np  # noqa: E402

NORM = {"bf16": 3e-3, "f32": 5e-6}


def ctx_of(H, dh, dtype, **kw):
    return fv.Context(hidden=H * dh, heads=H, head_dim=dh, ffn_hidden=256, dtype=dtype, **kw)


def empty_cache(B, heads, cap, dh, fill=0, **kw):
    full = lambda *s: torch.full(s, fill, dtype=torch.uint8, device="cuda")
    return fv.KVB(full(B, heads, cap, dh), full(B, heads, cap, dh), full(B, heads, -(-cap // 32)), full(B, heads, -(-cap // 32)), **kw)


def rows_of(seed, B, rows, heads, dh, dtype, spread=0.5):
    g = np.random.default_rng(seed)
    x = (g.standard_normal((B, rows, heads, dh)) * np.exp(g.normal(0, spread, (B, rows, heads, 1)))).astype(np.float32)
    return wl.round_to_bf16(x) if dtype == "bf16" else x


def load(kv, k, v):
    """Writes k, v [B, rows, heads, dh] by the oracle into the first rows of a cache; returns their values, head by head."""
    out = []
    for x, codes, scales in ((k, kv.k, kv.k_scale), (v, kv.v, kv.v_scale)):
        c, s = codes.cpu().numpy().copy(), scales.cpu().numpy().copy()
        kvb.append(c, s, [0] * x.shape[0], x)
        codes.copy_(torch.from_numpy(c))
        scales.copy_(torch.from_numpy(s))
        out.append(kvb.values(c, s)[:, :, :x.shape[1]])
    return out


def fill(kv, L):
    """Codes drawn as they are, with powers that differ from block to block, in the first rows of a cache; their values."""
    g, out = np.random.default_rng(11), []
    for codes, scales in ((kv.k, kv.k_scale), (kv.v, kv.v_scale)):
        c, s = codes.cpu().numpy().copy(), scales.cpu().numpy().copy()
        x = np.clip(g.standard_normal((*c.shape[:2], L, c.shape[3]), dtype=np.float32) * 100, -448, 448)
        c[:, :, :L] = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
        s[:, :, :-(-L // 32)] = g.integers(119, 122, (*s.shape[:2], -(-L // 32)))
        codes.copy_(torch.from_numpy(c))
        scales.copy_(torch.from_numpy(s))
        out.append(kvb.values(c[:, :, :L], s))
    return out


def attend(ctx, q, kv, dtype, B, n, junk=float("nan"), weights=None, **kw):
    o = torch.full((B, n, ctx.heads, ctx.head_dim), junk, dtype=tdtype(dtype), device="cuda")
    size = fv.fvar_kvb_attention_workspace_bytes(ctx, kv, B, n, weights is not None)
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")           # NaN in every float
    fv.fvar_kvb_attention(ctx, q, kv, B, n, o, ws, weights=weights, **kw)
    return o


def check(tag, got, want, dtype):
    got = to_np(got).astype(np.float64)
    norm = np.linalg.norm(got - want) / max(np.linalg.norm(want), 1e-30)
    worst = rel_err(got, want)
    print(f"[kvb] {tag}: norm {norm:.3g} max {worst:.3g}", flush=True)
    assert norm <= NORM[dtype] and worst <= TOL[dtype], (tag, norm, worst)


def check_weights(tag, got, want, q, k, scale):
    """got, want [B, heads, L]; q [B, n, H, dh], k [B, heads, L, dh]."""
    H, heads, dh = q.shape[2], k.shape[1], q.shape[3]
    most = max(float((np.abs(q[:, :, h].astype(np.float64)) @ np.abs(np.nan_to_num(k[:, h // (H // heads)])).swapaxes(-1, -2)).max()) for h in range(H))
    room = (2 * dh * 2.0 ** -24 * scale * most + 2.0 ** -20 + 2.0 ** -18) * want
    off = np.abs(got.cpu().numpy() - want)
    print(f"[kvb] {tag}: weights off by {float((off / np.maximum(want, 1e-30)).max()):.3g} of themselves", flush=True)
    assert (off <= room + 1e-30).all(), (tag, float((off - room).max()))


# ------------------------------------------------------------------------------------ writing and reading back
def _awkward_rows(dtype):
    """Blocks of 32 rows that a quantiser can get wrong, [blocks * 32, 64]."""
    g = np.random.default_rng(9)
    pick = lambda size: np.resize(np.concatenate([size * kvb.MIDS, -size * kvb.MIDS, size * kvb.VALUES, size * kvb.MIDS * 1.001]), (32, 64))
    blocks = [np.zeros((32, 64)), -np.zeros((32, 64))]
    for top in (448.0, 450.0, 464.0, 466.0, 224.0, 232.0, 234.0):
        x = g.standard_normal((32, 64))
        x[7, 9] = -top
        blocks.append(x)
    for e in (-126, -120, -118, -117, -116, -60, 0, 60, 118, 119):
        with np.errstate(over="ignore"):
            x = np.clip(pick(2.0 ** e), -3e38, 3e38)
        x[0, 0] = min(460.0 * 2.0 ** e, 3e38)
        blocks.append(x)
    x = g.standard_normal((32, 64))
    x[0, 0], x[3, 3], x[31, 63] = 3.3e38, -3.2e38, 1e-38
    blocks.append(x)
    for bad in (np.inf, -np.inf, np.nan):
        x = g.standard_normal((32, 64)) * 3
        x[5, 6], x[5, 7], x[20, 63] = bad, 1e3, -bad
        blocks.append(x)
    blocks.append(np.full((32, 64), np.nan))
    blocks.append(g.standard_normal((32, 64)) * np.exp(g.normal(0, 8, (32, 64))))
    x = np.concatenate(blocks).astype(np.float32)
    if dtype == "bf16":
        fine = np.isfinite(x)
        x = np.where(fine, wl.round_to_bf16(np.where(fine, x, 0)), x).astype(np.float32)
        x[np.isinf(x) & fine] = 3.3895313892515355e38
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("before", [0, 1, 33])
def test_append_is_the_definition_on_awkward_blocks(dtype, dh, before):
    x = _awkward_rows(dtype)
    x = np.concatenate([x, x[::-1]], axis=1)[:, :dh].reshape(1, -1, 1, dh)
    rows = x.shape[1]
    ctx, kv = ctx_of(1, dh, dtype), empty_cache(1, 1, before + rows + 2, dh, fill=0x41, len=before)
    xd = torch.from_numpy(x).cuda().to(tdtype(dtype))
    want = []
    for y, codes, scales in ((x, kv.k, kv.k_scale), (-x, kv.v, kv.v_scale)):
        want.append((codes.cpu().numpy().copy(), scales.cpu().numpy().copy()))
        kvb.append(*want[-1], [before], y)
    fv.fvar_kvb_append(ctx, kv, xd, -xd, 1, rows)
    for (c, s), codes, scales in zip(want, (kv.k, kv.v), (kv.k_scale, kv.v_scale)):
        assert np.array_equal(scales.cpu().numpy(), s)
        assert np.array_equal(codes.cpu().numpy(), c)
    kv.len = before + rows
    k, v = torch.empty_like(xd), torch.empty_like(xd)
    fv.fvar_kvb_read(ctx, kv, 1, before, rows, k, v)
    for got, (c, s) in zip((k, v), want):
        back = kvb.values(c, s)[:, :, before:before + rows].swapaxes(1, 2)
        assert np.array_equal(to_np(got), back.astype(np.float32), equal_nan=True)


@pytest.mark.parametrize("dtype,H,heads,dh,B,rows,before,cap", [
    ("bf16", 2, 2, 64, 1, 1, 0, 1), ("bf16", 4, 1, 128, 3, 1, 7, 9), ("bf16", 30, 30, 64, 2, 31, 5, 40), ("bf16", 16, 16, 128, 2, 33, 63, 96),
    ("bf16", 8, 2, 128, 5, 257, 1, 300), ("f32", 3, 3, 64, 2, 17, 3, 20), ("f32", 8, 4, 128, 1, 100, 28, 128), ("f32", 1, 1, 64, 1, 1, 4, 5)])
def test_append_and_read_back(dtype, H, heads, dh, B, rows, before, cap):
    ctx, kv = ctx_of(H, dh, dtype), empty_cache(B, heads, cap, dh, fill=0x5A)
    k0, v0 = rows_of(3, B, before, heads, dh, dtype), rows_of(4, B, before, heads, dh, dtype)
    if before:
        load(kv, 0.01 * k0, 0.01 * v0)                        # smaller than what comes, so that a shared block's power rises
    kv.len = before
    k, v = rows_of(1, B, rows, heads, dh, dtype), rows_of(2, B, rows, heads, dh, dtype)
    want = []
    for x, codes, scales in ((k, kv.k, kv.k_scale), (v, kv.v, kv.v_scale)):
        c, s = codes.cpu().numpy().copy(), scales.cpu().numpy().copy()
        kvb.append(c, s, [before] * B, x)
        want.append((c, s, kvb.values(c, s).swapaxes(1, 2).astype(np.float32)))
    fv.fvar_kvb_append(ctx, kv, to_dev(k, dtype), to_dev(v, dtype), B, rows)
    for (c, s, _), codes, scales in zip(want, (kv.k, kv.v), (kv.k_scale, kv.v_scale)):
        assert np.array_equal(codes.cpu().numpy(), c) and np.array_equal(scales.cpu().numpy(), s)
    kv.len = before + rows
    out = lambda r: torch.full((B, r, heads, dh), float("nan"), dtype=tdtype(dtype), device="cuda")
    for first, count in ((0, before + rows), (-rows, rows), (before, rows)):
        kb, vb = out(count), out(count)
        fv.fvar_kvb_read(ctx, kv, B, first, count, kb, vb)
        at = slice(before + rows + first, None) if first < 0 else slice(first, first + count)
        for got, (_, _, values) in zip((kb, vb), want):
            assert np.array_equal(to_np(got), values[:, :before + rows][:, at])
    kb, vb = out(rows), out(rows)
    fv.fvar_kvb_read(ctx, kv, B, -rows, rows, k=kb)
    fv.fvar_kvb_read(ctx, kv, B, -rows, rows, v=vb)
    assert np.array_equal(to_np(kb), want[0][2][:, before:before + rows]) and np.array_equal(to_np(vb), want[1][2][:, before:before + rows])
    if before + rows < cap:                                   # rows that are not held read as 0
        kb, vb = out(cap - before - rows), out(cap - before - rows)
        fv.fvar_kvb_read(ctx, kv, B, before + rows, cap - before - rows, kb, vb)
        assert not to_np(kb).any() and not to_np(vb).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_appended_one_by_one(dtype):
    """A token at a time, each row larger than the ones before: a block's power rises again and again."""
    H, heads, dh, B, cap = 4, 2, 64, 2, 70
    ctx, kv = ctx_of(H, dh, dtype), empty_cache(B, heads, cap, dh, fill=0x99)
    want = [(kv.k.cpu().numpy().copy(), kv.k_scale.cpu().numpy().copy()), (kv.v.cpu().numpy().copy(), kv.v_scale.cpu().numpy().copy())]
    for i in range(cap):
        k, v = (wl.round_to_bf16(rows_of(10 * i + j, B, 1, heads, dh, dtype) * np.float32(1.4 ** (i % 32))) for j in range(2))
        kv.len = i
        fv.fvar_kvb_append(ctx, kv, to_dev(k, dtype), to_dev(v, dtype), B, 1)
        kvb.append(*want[0], [i] * B, k)
        kvb.append(*want[1], [i] * B, v)
    for (c, s), codes, scales in zip(want, (kv.k, kv.v), (kv.k_scale, kv.v_scale)):
        assert np.array_equal(codes.cpu().numpy(), c) and np.array_equal(scales.cpu().numpy(), s)


def test_lengths_of_each_sample_and_rows_outside_the_cache():
    H, heads, dh, B, rows, cap = 4, 2, 128, 6, 40, 100
    lens = [0, 31, 90, 100, -5, 64]
    ctx = ctx_of(H, dh, "bf16")
    kv = empty_cache(B, heads, cap, dh, fill=0x33, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    fused = rows_of(1, B, rows, 3 * heads, dh, "bf16")
    want = []
    for x, codes, scales in ((fused[:, :, :heads], kv.k, kv.k_scale), (fused[:, :, 2 * heads:], kv.v, kv.v_scale)):
        want.append((codes.cpu().numpy().copy(), scales.cpu().numpy().copy()))
        kvb.append(*want[-1], lens, x)
    fd = to_dev(fused, "bf16")
    fv.fvar_kvb_append(ctx, kv, fd[:, :, :heads], fd[:, :, 2 * heads:], B, rows)       # parts of a fused projection's rows
    for (c, s), codes, scales in zip(want, (kv.k, kv.v), (kv.k_scale, kv.v_scale)):
        assert np.array_equal(codes.cpu().numpy(), c) and np.array_equal(scales.cpu().numpy(), s)
    kv.lens = torch.tensor([40, 71, 100, 100, 0, 100], dtype=torch.int32, device="cuda")
    k = torch.full((B, 50, heads, dh), float("nan"), dtype=torch.bfloat16, device="cuda")
    fv.fvar_kvb_read(ctx, kv, B, -50, 50, k=k)
    values = kvb.values(*want[0]).swapaxes(1, 2).astype(np.float32)
    for b, end in enumerate([40, 71, 100, 100, 0, 100]):
        at = np.arange(end - 50, end)
        assert np.array_equal(to_np(k)[b], np.where((at >= 0)[:, None, None], values[b][np.maximum(at, 0)], 0))


# ------------------------------------------------------------------------------------ attention
SHAPES = [("bf16", 2, 2, 64, 1, 1, 1), ("bf16", 4, 1, 128, 2, 1, 33), ("bf16", 16, 16, 128, 1, 1, 1300), ("bf16", 32, 8, 128, 3, 1, 517),
          ("bf16", 30, 30, 64, 2, 7, 100), ("bf16", 30, 10, 64, 1, 37, 95), ("bf16", 16, 16, 128, 2, 130, 333), ("bf16", 8, 2, 128, 1, 300, 64),
          ("bf16", 4, 4, 64, 3, 257, 700), ("bf16", 2, 1, 128, 1, 1000, 1500), ("f32", 4, 4, 64, 2, 1, 40), ("f32", 6, 2, 128, 1, 19, 129),
          ("f32", 16, 16, 64, 2, 128, 552), ("f32", 2, 1, 128, 2, 65, 1000)]
# three wavefronts per SIMD; whole rounds of workgroups and a divided rest; more keys per workgroup than it holds scale bytes of at once; the
# same with a single query; one query of few keys by eight wavefronts; fp32 in shares
LARGE = [("bf16", 30, 30, 64, 32, 200, 70), ("bf16", 16, 16, 128, 33, 129, 1030), ("bf16", 16, 16, 64, 4, 512, 4500), ("bf16", 16, 4, 128, 2, 3, 9000),
         ("bf16", 16, 16, 64, 1, 1, 700), ("f32", 4, 2, 64, 1, 5, 3000)]
# two groups of wavefronts, blocks of rows divided into shares; groups of four wavefronts in shares; blocks of rows that are not full
TILES = [("bf16", 2, 1, 128, 1, 1000, 6000), ("bf16", 8, 8, 64, 2, 600, 1700), ("bf16", 16, 16, 64, 5, 230, 4100), ("bf16", 16, 4, 64, 40, 40, 900)]
# blocks of 16 rows by a single wavefront, and by two
FEW = [("bf16", 16, 16, 128, 32, 64, 150), ("bf16", 16, 16, 64, 16, 64, 500), ("f32", 16, 16, 64, 40, 60, 90), ("f32", 16, 16, 64, 16, 70, 200),
       ("bf16", 16, 16, 128, 8, 400, 60), ("f32", 8, 4, 128, 20, 110, 31), ("bf16", 30, 30, 64, 9, 370, 26), ("bf16", 16, 16, 128, 17, 40, 55), ("bf16", 32, 16, 128, 16, 150, 64)]


@pytest.mark.parametrize("dtype,H,heads,dh,B,n,L", SHAPES + LARGE + TILES + FEW)
@pytest.mark.parametrize("kind", ["plain", "ragged", "masked"])
def test_attention_and_weights(dtype, H, heads, dh, B, n, L, kind):
    g = np.random.default_rng(L + n)
    cap = L + 5
    ctx, kv = ctx_of(H, dh, dtype), empty_cache(B, heads, cap, dh, fill=0x7F)           # NaN wherever nothing is written
    k, v = load(kv, rows_of(1, B, L, heads, dh, dtype), rows_of(2, B, L, heads, dh, dtype)) if B * L * heads < 3e5 else fill(kv, L)
    q = rows_of(3, B, n, H, dh, dtype, spread=0.2)
    lens, mask = [L] * B, None
    kv.len = L
    if kind == "ragged":
        lens = [L - b * (L // max(B, 1)) for b in range(B)] if B > 1 else [max(1, L // 2)]
        kv.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    if kind == "masked":
        mask = (g.random((B, cap)) < 0.7).astype(np.uint8) * 255
        mask[0, :L // 2] = 0
        kv.mask = torch.from_numpy(mask).cuda()
        hidden = torch.from_numpy(mask[:, :L] == 0).cuda()
        kv.k[:, :, :L][hidden[:, None].expand(B, heads, L)] = 0x7F             # what hidden rows hold has no influence
        kv.v[:, :, :L][hidden[:, None].expand(B, heads, L)] = 0xFF
    want, w = kvb.attention(q, k, v, 1 / math.sqrt(dh), lens, None if mask is None else mask[:, :L])
    tag = f"{dtype} {H}/{heads}x{dh} B{B} n{n} L{L} {kind}"
    qd = to_dev(q, dtype)
    o = attend(ctx, qd, kv, dtype, B, n)
    check(tag, o, want, dtype)
    got = torch.full((B, heads, cap), 3.0, device="cuda")
    o2 = attend(ctx, qd, kv, dtype, B, n, weights=got)
    assert torch.equal(o, o2)
    check_weights(tag, got[:, :, :L][:, :, :], np.where((np.arange(L) < np.array(lens)[:, None])[:, None], w, 3.0), q, k, 1 / math.sqrt(dh))
    assert (got[:, :, L:] == 3).all()
    again = got.clone()
    attend(ctx, qd, kv, dtype, B, n, weights=again, add=True)
    held = torch.arange(cap, device="cuda") < torch.tensor(lens, device="cuda")[:, None, None]
    assert torch.equal(again, torch.where(held, got + got, got))               # the same sums, once more


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("junk", [0, 255])
@pytest.mark.parametrize("H,heads,dh,B,n", [(4, 2, 64, 2, 1), (2, 2, 128, 1, 9), (8, 8, 64, 1, 40), (8, 4, 128, 2, 150), (30, 30, 64, 32, 200), (16, 16, 128, 33, 129)])
def test_scales_of_blocks_that_hold_nothing_have_no_influence(dtype, junk, H, heads, dh, B, n):
    """Lengths at which tiles of two blocks, or of 256 keys, end in blocks that were never written, whatever stands there."""
    if dtype == "f32" and B * n > 500:
        return
    cap = 640
    ctx = ctx_of(H, dh, dtype)
    x, q = [rows_of(s, B, 353, heads, dh, dtype) for s in (1, 2)], to_dev(rows_of(3, B, n, H, dh, dtype, spread=0.2), dtype)
    a, b = empty_cache(B, heads, cap, dh, fill=127), empty_cache(B, heads, cap, dh, fill=junk)
    for L in (1, 32, 65, 96, 353):
        for kv in (a, b):
            kv.len, kv.lens = 0, None
            for t in (kv.k, kv.v, kv.k_scale, kv.v_scale):
                t.fill_(junk if kv is b else 127)
            fv.fvar_kvb_append(ctx, kv, *[to_dev(np.ascontiguousarray(y[:, :L]), dtype) for y in x], B, L)
            kv.len = L
        for ragged in (False, True):
            outs = []
            for kv in (a, b):
                kv.lens = torch.full((B,), L, dtype=torch.int32, device="cuda") if ragged else None
                w = torch.zeros((B, heads, cap), device="cuda")
                outs.append((attend(ctx, q, kv, dtype, B, n, weights=w), w))
            assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1]), (L, ragged)
            assert torch.isfinite(outs[0][0]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_without_a_visible_row(dtype):
    H, heads, dh, B, n, cap = 4, 2, 64, 3, 200, 96
    ctx, kv = ctx_of(H, dh, dtype), empty_cache(B, heads, cap, dh, fill=0x7F, lens=torch.tensor([0, 96, -3], dtype=torch.int32, device="cuda"))
    load(kv, rows_of(1, B, cap, heads, dh, dtype), rows_of(2, B, cap, heads, dh, dtype))
    kv.mask = torch.zeros((B, cap), dtype=torch.bool, device="cuda")
    w = torch.full((B, heads, cap), 2.0, device="cuda")
    for rows in (n, 1):
        o = attend(ctx, to_dev(rows_of(3, B, rows, H, dh, dtype), dtype), kv, dtype, B, rows, weights=w)
        assert not to_np(o).any()
    assert (w[0] == 2).all() and (w[1] == 0).all() and (w[2] == 2).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 150])
@pytest.mark.parametrize("size", [1e-3, 30.0, 1e10])
def test_attention_over_scores_of_every_size(dtype, n, size):
    """Scores up to 10^11: weights are 1 or 0 then, and the output is the value of the best key."""
    H, heads, dh, B, L = 2, 2, 128, 1, 300
    ctx, kv = ctx_of(H, dh, dtype), empty_cache(B, heads, L, dh, len=L)
    k, v = load(kv, rows_of(1, B, L, heads, dh, dtype), rows_of(2, B, L, heads, dh, dtype))
    q = rows_of(3, B, n, H, dh, dtype, spread=0.1) * np.float32(size)
    q = wl.round_to_bf16(q) if dtype == "bf16" else q
    want, w = kvb.attention(q, k, v, 1 / math.sqrt(dh), [L])
    got = torch.zeros((B, heads, L), device="cuda")
    o = attend(ctx, to_dev(q, dtype), kv, dtype, B, n, weights=got)
    if size > 1e3:                                            # rows of queries whose best two scores differ by more than fp32 can hold apart
        s = np.stack([q[0, :, h].astype(np.float64) @ k[0, h].T for h in range(H)], 1) / math.sqrt(dh)
        two = np.sort(s, -1)[..., -2:]
        clear = two[..., 1] - two[..., 0] > 50 + 2 * dh * 2.0 ** -24 * np.abs(q[0].astype(np.float64)).max() * np.abs(k).max() * dh
        assert clear.any()
        assert rel_err(to_np(o)[0][clear], want[0][clear]) <= (2.0 ** -8 if dtype == "bf16" else 1e-6)
        assert np.isfinite(to_np(o)).all() and torch.isfinite(got).all()
        return
    if size < 1:                                              # (scores of up to 100 times 30 carry fp32's error of them into every weight)
        check(f"{dtype} n{n} size {size}", o, want, dtype)
    else:
        assert np.linalg.norm(to_np(o) - want) <= NORM["bf16"] * np.linalg.norm(want)
    check_weights(f"{dtype} n{n} size {size}", got, w, q, k, 1 / math.sqrt(dh))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 140])
@pytest.mark.parametrize("e", [-100, -40, -17, -9, 9, 40, 100])
def test_attention_over_values_of_every_size(dtype, n, e):
    """Blocks of values of very different sizes, the largest first and last: the sums are rescaled, and small blocks count down to 2^-19 of the
    largest with all their bits."""
    H, heads, dh, B, L = 2, 1, 64, 2, 160
    ctx, kv = ctx_of(H, dh, dtype), empty_cache(B, heads, L, dh, len=L)
    x = rows_of(2, B, L, heads, dh, dtype)
    x[:, 64:96] *= np.float32(2.0 ** e)
    k, v = load(kv, rows_of(1, B, L, heads, dh, dtype), x)
    q = rows_of(3, B, n, H, dh, dtype, spread=0.2)
    want, _ = kvb.attention(q, k, v, 1 / math.sqrt(dh), [L] * B)
    check(f"{dtype} n{n} values 2^{e}", attend(ctx, to_dev(q, dtype), kv, dtype, B, n), want, dtype)


@pytest.mark.parametrize("n", [1, 40, 300])
def test_queries_that_are_no_numbers_keep_to_their_rows(n):
    H, heads, dh, B, L = 2, 2, 64, 1, 200
    ctx, kv = ctx_of(H, dh, "bf16"), empty_cache(B, heads, L, dh, len=L)
    load(kv, rows_of(1, B, L, heads, dh, "bf16"), rows_of(2, B, L, heads, dh, "bf16"))
    q = to_dev(rows_of(3, B, n, H, dh, "bf16"), "bf16")
    w, clean = torch.zeros((B, heads, L), device="cuda"), torch.zeros((B, heads, L), device="cuda")
    want = attend(ctx, q, kv, "bf16", B, n)
    q[0, 0, 0, 5] = float("nan")
    q[0, n - 1, 1, 60] = float("inf")
    o = attend(ctx, q, kv, "bf16", B, n, weights=w)
    assert torch.isnan(o[0, 0, 0]).all() and torch.isnan(o[0, n - 1, 1]).all()
    same = torch.ones((n, H), dtype=torch.bool)
    same[0, 0] = same[n - 1, 1] = False
    assert torch.equal(o[0][same.cuda()], want[0][same.cuda()])
    if n > 1:
        assert torch.isfinite(w).all() and abs(float(w[0, 0].sum()) - (n - 1)) < 1e-3 and abs(float(w[0, 1].sum()) - (n - 1)) < 1e-3


def test_attention_takes_rows_of_a_fused_projection_and_other_streams_and_graphs():
    H, heads, dh, B, n, L = 8, 4, 128, 2, 50, 400
    ctx, kv = ctx_of(H, dh, "bf16"), empty_cache(B, heads, L, dh, len=L)
    load(kv, rows_of(1, B, L, heads, dh, "bf16"), rows_of(2, B, L, heads, dh, "bf16"))
    fused = to_dev(rows_of(3, B, n, H + 2 * heads, dh, "bf16"), "bf16")
    want, got = torch.zeros((B, heads, L), device="cuda"), torch.zeros((B, heads, L), device="cuda")
    o = attend(ctx, fused[:, :, :H].contiguous(), kv, "bf16", B, n, weights=want)
    assert torch.equal(o, attend(ctx, fused[:, :, :H], kv, "bf16", B, n, weights=got)) and torch.equal(want, got)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ws = torch.empty(fv.fvar_kvb_attention_workspace_bytes(ctx, kv, B, n, True), dtype=torch.uint8, device="cuda")
    o2 = torch.empty_like(o)
    got.zero_()
    side.wait_stream(torch.cuda.current_stream())
    fv.fvar_kvb_attention(ctx, fused[:, :, :H], kv, B, n, o2, ws, weights=got, stream=side)
    side.synchronize()
    assert torch.equal(o, o2) and torch.equal(want, got)
    # a step in a graph: rows appended at a length that the GPU holds, attention over it, replayed as the length grows
    kv = empty_cache(B, heads, L, dh, lens=torch.zeros(B, dtype=torch.int32, device="cuda"))
    step, k, v = fused[:, :1, :H], fused[:, :1, H:H + heads], fused[:, :1, H + heads:]
    x = torch.empty((B, 1, H + 2 * heads, dh), dtype=torch.bfloat16, device="cuda")
    o3, w = torch.empty((B, 1, H, dh), dtype=torch.bfloat16, device="cuda"), torch.zeros((B, heads, L), device="cuda")
    ws = torch.empty(fv.fvar_kvb_attention_workspace_bytes(ctx, kv, B, 1, True), dtype=torch.uint8, device="cuda")

    def one(cache, out, weights):
        fv.fvar_kvb_append(ctx, cache, x[:, :, H:H + heads], x[:, :, H + heads:], B, 1)
        cache.lens.add_(1)
        fv.fvar_kvb_attention(ctx, x[:, :, :H], cache, B, 1, out, ws, weights=weights, add=True)

    x.copy_(fused[:, :1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one(kv, o3, w)
    kv.lens.zero_()
    w.zero_()
    eager, w2, o4 = empty_cache(B, heads, L, dh, lens=torch.zeros(B, dtype=torch.int32, device="cuda")), torch.zeros_like(w), torch.empty_like(o3)
    for i in range(40):
        x.copy_(fused[:, i:i + 1])
        graph.replay()
        one(eager, o4, w2)
        torch.cuda.synchronize()
        assert torch.equal(o3, o4) and torch.equal(w, w2) and torch.equal(kv.k, eager.k) and torch.equal(kv.v_scale, eager.v_scale)
    assert kv.lens.tolist() == [40, 40]


def test_cache_whose_offsets_pass_32_bits():
    """Two samples of 9 heads over 2^21 rows: 4.8 GB of keys and as much of values, of which the mask leaves the last 100 rows or so."""
    B, heads, dh, cap, rows = 2, 9, 128, 2 ** 21 + 33, 30
    start, lens = 2 ** 21 - 96, [cap - 70, cap - 40]
    ctx, kv = ctx_of(heads, dh, "bf16"), empty_cache(B, heads, cap, dh, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    k, v = rows_of(1, B, rows, heads, dh, "bf16"), rows_of(2, B, rows, heads, dh, "bf16")
    tail, powers = slice(start, cap), slice(start // 32, None)
    want = []
    for codes, scales, x in ((kv.k, kv.k_scale, k), (kv.v, kv.v_scale, v)):
        codes[:, :, tail].random_(0, 127)
        scales[:, :, powers].random_(118, 122)
        want.append((codes[:, :, tail].cpu().numpy().copy(), scales[:, :, powers].cpu().numpy().copy()))
        kvb.append(*want[-1], [n - start for n in lens], x)
    fv.fvar_kvb_append(ctx, kv, to_dev(k, "bf16"), to_dev(v, "bf16"), B, rows)
    kv.lens.add_(rows)
    lens = [n + rows - start for n in lens]
    for codes, scales, (c, s) in ((kv.k, kv.k_scale, want[0]), (kv.v, kv.v_scale, want[1])):
        assert np.array_equal(codes[:, :, tail].cpu().numpy(), c) and np.array_equal(scales[:, :, powers].cpu().numpy(), s)
    held = [kvb.values(c, s) for c, s in want]
    back = [torch.empty((B, rows, heads, dh), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    fv.fvar_kvb_read(ctx, kv, B, -rows, rows, *back)
    for got, x in zip(back, held):
        assert np.array_equal(to_np(got), np.stack([x[b, :, n - rows:n] for b, n in enumerate(lens)]).swapaxes(1, 2))
    kv.mask = torch.zeros((B, cap), dtype=torch.uint8, device="cuda")
    kv.mask[:, start + 10:] = 1
    kv.mask[1, start + 50] = 0
    mask = kv.mask[:, tail].cpu().numpy()
    for n in (1, 200):
        q = rows_of(3, B, n, heads, dh, "bf16", spread=0.2)
        o, w = kvb.attention(q, *held, dh ** -0.5, lens, mask)
        got = torch.full((B, heads, cap), 3.0, device="cuda")
        check(f"long, n{n}", attend(ctx, to_dev(q, "bf16"), kv, "bf16", B, n, weights=got), o, "bf16")
        there = (np.arange(cap - start) < np.array(lens)[:, None])[:, None]
        check_weights(f"long, n{n}", got[:, :, tail], np.where(there, w, 3.0), q, held[0], dh ** -0.5)
        assert not got[:, :, :start].any()
    keep, weights = 64, got[:, :, tail].cpu().numpy()
    outs = [kvb.evict(c, s, weights, lens, keep, 5, mask) for c, s in want]
    to, tw = empty_cache(B, heads, keep, dh), torch.empty((B, heads, keep), device="cuda")
    count, idx = torch.empty(B, dtype=torch.int32, device="cuda"), torch.empty((B, heads, keep), dtype=torch.int32, device="cuda")
    ws = torch.empty(fv.fvar_kvb_evict_workspace_bytes(ctx, kv, B, keep), dtype=torch.uint8, device="cuda")
    fv.fvar_kvb_evict(ctx, kv, got, B, keep, 5, to, tw, count, idx, ws)
    assert np.array_equal(idx.cpu().numpy(), outs[0][0] + start) and count.tolist() == [keep, keep]
    assert np.array_equal(tw.cpu().numpy(), np.take_along_axis(weights, outs[0][0], -1))
    fv.fvar_kvb_evict(ctx, kv, got, B, keep, 5, kv, got, kv.lens, idx, ws)       # in place: the same rows at the front
    for codes, scales, codes2, scales2, out in ((to.k, to.k_scale, kv.k, kv.k_scale, outs[0]), (to.v, to.v_scale, kv.v, kv.v_scale, outs[1])):
        assert np.array_equal(codes.cpu().numpy(), np.array([[h[0] for h in b] for b in out[2]]))
        assert np.array_equal(scales.cpu().numpy(), np.array([[h[1] for h in b] for b in out[2]]))
        assert torch.equal(codes, codes2[:, :, :keep]) and torch.equal(scales, scales2[:, :, :keep // 32])
    assert torch.equal(got[:, :, :keep], tw) and not got[:, :, keep:].any()


def test_debug_checks_look_at_lengths():
    H, dh, B, cap = 2, 64, 2, 40
    ctx, kv = ctx_of(H, dh, "bf16"), empty_cache(B, H, cap, dh, lens=torch.tensor([3, 41], dtype=torch.int32, device="cuda"))
    x = to_dev(rows_of(1, B, 1, H, dh, "bf16"), "bf16")
    fv.fvar_debug_checks(ctx, True)
    with pytest.raises(fv.FvarError) as e:
        fv.fvar_kvb_append(ctx, kv, x, x, B, 1)
    assert e.value.status == fv.FVAR_ERR_INVALID_ARG
    kv.lens = torch.tensor([3, 39], dtype=torch.int32, device="cuda")
    fv.fvar_kvb_append(ctx, kv, x, x, B, 1)


# ------------------------------------------------------------------------------------ the block
@pytest.mark.parametrize("dtype,d,H,B,M,keep,Lp,ragged,turned,weigh", [
    ("bf16", 256, 4, 2, 40, 40, 30, False, True, True), ("bf16", 256, 2, 2, 100, 37, 65, True, True, True), ("bf16", 512, 8, 1, 300, 300, 100, False, False, True),
    ("f32", 256, 4, 2, 64, 20, 33, True, True, False), ("f32", 256, 2, 1, 50, 50, 0, False, False, False), ("bf16", 1024, 8, 3, 256, 130, 200, False, True, True)])
def test_block_over_the_cache(dtype, d, H, B, M, keep, Lp, ragged, turned, weigh):
    """The block with W_o = 1 and an MLP of 0 gives x + attention: against the oracle's attention over the cache that the block left, whose
    new rows are the oracle's of the plain block's K and V rows, turned by the call of their own."""
    dh, F = d // H, 64
    x = wl.activations_lowrank(B, M, d, seed=100 + M, bf16=dtype == "bf16")
    g = np.random.default_rng(101)
    bf = lambda a: wl.round_to_bf16(a) if dtype == "bf16" else a.astype(np.float32)
    w = {"w_qkv": bf(0.05 * g.standard_normal((3 * d, d))), "b_qkv": bf(0.1 * g.standard_normal(3 * d)), "w_o": np.eye(d, dtype=np.float32),
         "w_fc1": np.zeros((F, d), np.float32), "w_fc2": np.zeros((d, F), np.float32)}
    wd = {n: to_dev(a, dtype) for n, a in w.items()}
    rolled = dict(wd, w_qkv=wd["w_qkv"].roll(d, 0).contiguous(), b_qkv=wd["b_qkv"].roll(d, 0).contiguous())   # q rows come out as K rows
    ctx = fv.Context(hidden=d, heads=H, head_dim=dh, ffn_hidden=F, dtype=dtype)
    xd = to_dev(x, dtype)
    idx = np.stack([np.sort(g.permutation(M)[:keep]) for _ in range(B)]).astype(np.int32)
    idx_d = torch.from_numpy(idx).cuda()
    cap = Lp + keep + 2

    def plain(weights):
        K, V = (torch.zeros((B, cap, H, dh), dtype=tdtype(dtype), device="cuda") for _ in range(2))
        y = torch.empty((B, keep, d), dtype=tdtype(dtype), device="cuda")
        ws = torch.empty(fv.fvar_block_workspace_bytes(ctx, B, keep), dtype=torch.uint8, device="cuda")
        fv.fvar_block_forward_pruned(ctx, weights, xd, B, M, idx_d, keep, K, V, cap, Lp, y, ws)
        return K[:, Lp:Lp + keep].contiguous(), V[:, Lp:Lp + keep].contiguous()

    (kn, vn), (qn, _) = plain(wd), plain(rolled)
    r = fv.Rope(dim=32, axes=2, interleaved=True) if turned else None
    pos = torch.from_numpy(np.stack([idx // 16, idx % 16], -1).astype(np.int32)).cuda() if turned else None
    if turned:
        fv.fvar_rope_apply(ctx, r, pos, B, keep, qn, kn)
    qn, kn, vn = to_np(qn), to_np(kn), to_np(vn)
    lens = [Lp - 9 * b for b in range(B)] if ragged else [Lp] * B
    kv = empty_cache(B, H, cap, dh, len=Lp, lens=torch.tensor(lens, dtype=torch.int32, device="cuda") if ragged else None)
    if Lp:
        load(kv, rows_of(102, B, Lp, H, dh, dtype), rows_of(103, B, Lp, H, dh, dtype))
    want = []
    for rows, codes, scales in ((kn, kv.k, kv.k_scale), (vn, kv.v, kv.v_scale)):
        want.append((codes.cpu().numpy().copy(), scales.cpu().numpy().copy()))
        kvb.append(*want[-1], lens, rows)
    fv.fvar_debug_checks(ctx, True)                           # with the canary behind the workspace
    size = fv.fvar_block_kvb_workspace_bytes(ctx, kv, B, keep, weights=weigh)
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    y = torch.empty((B, keep, d), dtype=tdtype(dtype), device="cuda")
    sums = torch.full((B, H, cap), 0.5, device="cuda") if weigh else None
    if keep == M:
        fv.fvar_block_forward_dense_kvb(ctx, wd, xd, B, M, kv, y, ws, rope=r, pos=pos, weights=sums, add=True)
    else:
        fv.fvar_block_forward_pruned_kvb(ctx, wd, xd, B, M, idx_d, keep, kv, y, ws, rope=r, pos=pos, weights=sums, add=True)
    fv.fvar_debug_checks(ctx, False)
    for (c, s), codes, scales in zip(want, (kv.k, kv.v), (kv.k_scale, kv.v_scale)):
        assert np.array_equal(codes.cpu().numpy(), c)
        assert np.array_equal(scales.cpu().numpy(), s)
    held = [kvb.values(c, s) for c, s in want]
    ends = [n + keep for n in lens]
    att, got = kvb.attention(qn, *held, dh ** -0.5, ends)
    xk = np.stack([x[b, idx[b]] for b in range(B)])
    check(f"block {dtype} {B}x{keep}", y, xk + att.reshape(B, keep, d), dtype)
    if weigh:
        there = (np.arange(cap) < np.array(ends)[:, None])[:, None]
        check_weights(f"block {dtype} {B}x{keep}", sums, np.where(there, 0.5 + got, 0.5), qn, held[0], dh ** -0.5)
