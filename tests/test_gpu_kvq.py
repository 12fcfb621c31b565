"""The 4-bit cache on the GPU through the C ABI, against its definition in 64 bits.

Writing and reading back are exact: codes and scales have to be the oracle's bit for bit.  Attention: the output is rounded
to bf16 once (2^-8 relative at most, 1.7e-3 rms), and on the way the probabilities and the queries to about as many bits, each an
independent error of the same size or less: 2-norm of the error at most 4e-3 of the result's; in fp32 sums of a
few thousand terms leave at most 5e-6.  The largest error of one element is held to the library's bars (2e-2, 1e-4 of
max(|o|, rms)); where all weights are equal or one is 1, to the rounding of the output alone."""
import numpy as np
import pytest
import torch

import paper_2512_16483_amd as fv
import workloads as wl
from oracle import kvq

pytestmark = pytest.mark.gpu

from gpu_util import TOL, rel_err, tdtype, to_dev, to_np  # noqa: E402

NORM = {"bf16": 4e-3, "f32": 5e-6}


def _ctx(H, dh, dtype, **kw):
    return fv.Context(hidden=H * dh, heads=H, head_dim=dh, ffn_hidden=256, dtype=dtype, **kw)


def _empty_cache(B, heads, cap, dh, fill=0, **kw):
    full = lambda *s: torch.full(s, fill, dtype=torch.uint8, device="cuda")
    return fv.KVQ(full(B, heads, cap, dh // 2), full(B, heads, cap, dh // 2), full(B, heads, cap, dh // 32),
                  full(B, heads, cap, dh // 32), **kw)


def _rows(seed, B, rows, heads, dh, dtype, spread=0.5):
    g = np.random.default_rng(seed)
    x = (g.standard_normal((B, rows, heads, dh)) * np.exp(g.normal(0, spread, (B, rows, heads, 1)))).astype(np.float32)
    return wl.round_to_bf16(x) if dtype == "bf16" else x


def _load(kv, k, v):
    """Quantises k, v [B, rows, heads, dh] by the oracle into the first rows of a cache; returns their values, head by head."""
    out = []
    for x, codes, scales in ((k, kv.k, kv.k_scale), (v, kv.v, kv.v_scale)):
        c, s = kvq.quantise(np.swapaxes(x, 1, 2))
        codes[:, :, :c.shape[2]] = torch.from_numpy(c).cuda()
        scales[:, :, :s.shape[2]] = torch.from_numpy(s).cuda()
        out.append(kvq.values(c, s))
    return out


def _attend(ctx, q, kv, dtype, B, n, junk=float("nan"), **kw):
    o = torch.full((B, n, ctx.heads, ctx.head_dim), junk, dtype=tdtype(dtype), device="cuda")
    size = fv.fvar_kvq_attention_workspace_bytes(ctx, kv, B, n)
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")           # NaN in every float
    fv.fvar_kvq_attention(ctx, q, kv, B, n, o, ws, **kw)
    return o


def _check(tag, got, want, dtype):
    got = to_np(got).astype(np.float64)
    norm = np.linalg.norm(got - want) / max(np.linalg.norm(want), 1e-30)
    worst = rel_err(got, want)
    print(f"[kvq] {tag}: norm {norm:.3g} max {worst:.3g}", flush=True)
    assert norm <= NORM[dtype] and worst <= TOL[dtype], (tag, norm, worst)


# ------------------------------------------------------------------------------------ writing and reading back
def _awkward_blocks(dtype):
    """Blocks of 32 that a quantiser can get wrong, as rows of 64."""
    mids = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0])
    pad = lambda x: np.concatenate([x, np.zeros(32 - len(x))])
    blocks = [np.zeros(32), -np.zeros(32)]
    for top in (6.0, 6.96875, 7.0, 7.03125, 4.0, 3.5):
        blocks += [pad(np.concatenate([mids[:6], -mids[:6], [top]])), pad(np.concatenate([mids[:6] * 0.99, mids[:6] * 1.01, [-top]]))]
    for e in (-126, -125, -124, -123, -120, -60, 60, 120, 124, 125):
        blocks.append(pad(np.concatenate([mids, [-0.0, 6.0]]) * 2.0 ** e))
    blocks += [pad([3.3e38, -1e38, 1.0]), pad([2.0 ** 127 * 1.9, 2.0 ** 126]), pad([2.0 ** 127 * 1.75]), pad([1e-45, -1e-40, 1e-38])]
    for bad in (np.inf, -np.inf, np.nan):
        blocks.append(pad([1.0, bad, -2.0]))
    if len(blocks) % 2:
        blocks.append(pad([1.0]))
    x = np.array(blocks).reshape(-1, 64).astype(np.float32)
    if dtype == "bf16":
        fine = np.isfinite(x)
        x = np.where(fine, wl.round_to_bf16(np.where(fine, x, 0)), x).astype(np.float32)
        x[np.isinf(x) & fine] = 3.3895313892515355e38
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 128])
def test_append_is_the_definition_on_awkward_blocks(dtype, dh):
    x = _awkward_blocks(dtype)
    x = np.concatenate([x, x[: (-len(x)) % (dh // 64)]]).reshape(1, -1, 1, dh)
    rows = x.shape[1]
    ctx, kv = _ctx(1, dh, dtype), _empty_cache(1, 1, rows + 2, dh, fill=0xA5, len=1)
    xd = torch.from_numpy(x).cuda().to(tdtype(dtype))
    assert dtype == "f32" or torch.equal(torch.nan_to_num(xd.float(), nan=-7.0), torch.nan_to_num(torch.from_numpy(x).cuda(), nan=-7.0))
    fv.fvar_kvq_append(ctx, kv, xd, -xd, 1, rows)
    for y, codes, scales in ((x, kv.k, kv.k_scale), (-x, kv.v, kv.v_scale)):
        c, s = kvq.quantise(np.swapaxes(y, 1, 2))
        assert np.array_equal(scales[:, :, 1:rows + 1].cpu().numpy(), s)
        assert np.array_equal(codes[:, :, 1:rows + 1].cpu().numpy(), c)
        for t in (codes, scales):                             # nothing beside the rows is touched
            assert (t[:, :, 0] == 0xA5).all() and (t[:, :, rows + 1:] == 0xA5).all()
    kv.len = rows + 1
    k, v = torch.empty_like(xd), torch.empty_like(xd)
    fv.fvar_kvq_read(ctx, kv, 1, 1, rows, k, v)
    for got, codes, scales in ((k, kv.k, kv.k_scale), (v, kv.v, kv.v_scale)):
        want = kvq.values(codes.cpu().numpy(), scales.cpu().numpy())[:, :, 1:rows + 1].swapaxes(1, 2)
        assert np.array_equal(to_np(got), want.astype(np.float32), equal_nan=True)


@pytest.mark.parametrize("dtype,H,heads,dh,B,rows,before,cap", [
    ("bf16", 2, 2, 64, 1, 1, 0, 1), ("bf16", 4, 1, 128, 3, 1, 7, 9), ("bf16", 30, 30, 64, 2, 31, 5, 40), ("bf16", 16, 16, 128, 2, 33, 63, 96),
    ("bf16", 8, 2, 128, 5, 257, 1, 300), ("f32", 3, 3, 64, 2, 17, 3, 20), ("f32", 8, 4, 128, 1, 100, 28, 128), ("f32", 1, 1, 64, 1, 1, 4, 5)])
def test_append_and_read_back(dtype, H, heads, dh, B, rows, before, cap):
    ctx, kv = _ctx(H, dh, dtype), _empty_cache(B, heads, cap, dh, fill=0x5A, len=before)
    k, v = _rows(1, B, rows, heads, dh, dtype), _rows(2, B, rows, heads, dh, dtype)
    fv.fvar_kvq_append(ctx, kv, to_dev(k, dtype), to_dev(v, dtype), B, rows)
    held = []
    for x, codes, scales in ((k, kv.k, kv.k_scale), (v, kv.v, kv.v_scale)):
        c, s = kvq.quantise(np.swapaxes(x, 1, 2))
        held.append(kvq.values(c, s).swapaxes(1, 2).astype(np.float32))
        assert np.array_equal(codes[:, :, before:before + rows].cpu().numpy(), c)
        assert np.array_equal(scales[:, :, before:before + rows].cpu().numpy(), s)
        for t in (codes, scales):
            assert (t[:, :, :before] == 0x5A).all() and (t[:, :, before + rows:] == 0x5A).all()
    kv.len = before + rows
    out = lambda r: torch.full((B, r, heads, dh), float("nan"), dtype=tdtype(dtype), device="cuda")
    for first in (before, -rows):
        kb, vb = out(rows), out(rows)
        fv.fvar_kvq_read(ctx, kv, B, first, rows, kb, vb)
        assert np.array_equal(to_np(kb), held[0]) and np.array_equal(to_np(vb), held[1])
    kb, vb = out(rows), out(rows)
    fv.fvar_kvq_read(ctx, kv, B, -rows, rows, k=kb)
    fv.fvar_kvq_read(ctx, kv, B, -rows, rows, v=vb)
    assert np.array_equal(to_np(kb), held[0]) and np.array_equal(to_np(vb), held[1])
    if before + rows < cap:                                   # rows that are not held read as 0
        kb, vb = out(cap - before - rows), out(cap - before - rows)
        fv.fvar_kvq_read(ctx, kv, B, before + rows, cap - before - rows, kb, vb)
        assert not to_np(kb).any() and not to_np(vb).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_by_lengths_of_each_sample(dtype):
    """Lengths of every kind: rows that would leave the capacity, or lie before it, are left out."""
    B, heads, dh, rows, cap = 6, 2, 64, 5, 12
    lens = [0, 7, 8, 12, -3, 2 ** 31 - 1]
    lens_d = torch.tensor(lens, dtype=torch.int32, device="cuda")
    ctx, kv = _ctx(heads, dh, dtype), _empty_cache(B, heads, cap, dh, fill=0x5A, lens=lens_d)
    k, v = _rows(3, B, rows, heads, dh, dtype), _rows(4, B, rows, heads, dh, dtype)
    fv.fvar_kvq_append(ctx, kv, to_dev(k, dtype), to_dev(v, dtype), B, rows)
    for x, codes, scales in ((k, kv.k, kv.k_scale), (v, kv.v, kv.v_scale)):
        c, s = kvq.quantise(np.swapaxes(x, 1, 2))
        want_c, want_s = np.full(tuple(codes.shape), 0x5A, np.uint8), np.full(tuple(scales.shape), 0x5A, np.uint8)
        for b in range(B):
            for j in range(rows):
                if 0 <= lens[b] + j < cap:
                    want_c[b, :, lens[b] + j], want_s[b, :, lens[b] + j] = c[b, :, j], s[b, :, j]
        assert np.array_equal(codes.cpu().numpy(), want_c) and np.array_equal(scales.cpu().numpy(), want_s)
    # read from the end of each sample's rows; lengths are held to the capacity
    out = torch.full((B, rows, heads, dh), float("nan"), dtype=tdtype(dtype), device="cuda")
    fv.fvar_kvq_read(ctx, kv, B, -rows, rows, k=out)
    held = kvq.values(kv.k.cpu().numpy(), kv.k_scale.cpu().numpy())
    for b in range(B):
        n = min(max(lens[b], 0), cap)
        want = np.zeros((rows, heads, dh))
        for j in range(rows):
            if n - rows + j >= 0:
                want[j] = held[b, :, n - rows + j]
        assert np.array_equal(to_np(out[b]), want.astype(np.float32))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 9])
def test_rows_of_a_fused_projection(dtype, rows):
    """k, v and q as parts of one [B, rows, q | k | v] tensor, on a stream of their own."""
    B, H, heads, dh = 3, 4, 2, 64
    width = (H + 2 * heads) * dh
    qkv = _rows(5, B, rows, H + 2 * heads, dh, dtype).reshape(B, rows, width)
    qkv_d = to_dev(qkv, dtype)
    q, k, v = qkv_d[..., :H * dh], qkv_d[..., H * dh:(H + heads) * dh], qkv_d[..., (H + heads) * dh:]
    ctx, kv = _ctx(H, dh, dtype), _empty_cache(B, heads, rows + 3, dh, len=0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    fv.fvar_kvq_append(ctx, kv, k, v, B, rows, stream=side)
    kv.len = rows
    with torch.cuda.stream(side):
        o = _attend(ctx, q, kv, dtype, B, rows)
    torch.cuda.current_stream().wait_stream(side)
    c = [kvq.values(*kvq.quantise(np.swapaxes(qkv[..., a:b].reshape(B, rows, heads, dh), 1, 2)))
         for a, b in ((H * dh, (H + heads) * dh), ((H + heads) * dh, width))]
    _check(f"fused {dtype} {rows}", o, kvq.attention(qkv[..., :H * dh].reshape(B, rows, H, dh), *c, dh ** -0.5, [rows] * B), dtype)
    with pytest.raises(ValueError):
        fv.fvar_kvq_append(ctx, kv, qkv_d[..., :heads * dh].transpose(0, 1), v, B, rows)


# ------------------------------------------------------------------------------------ attention
LENGTHS = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 1000]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh,H,heads", [(64, 6, 6), (64, 8, 2), (128, 4, 4), (128, 8, 1)])
@pytest.mark.parametrize("n", [1, 3, 17, 70])
def test_attention_at_every_kind_of_length(dtype, dh, H, heads, n):
    """One sample per length, in one cache: lengths around every tile's and block's end."""
    B, L = len(LENGTHS) + 1, max(LENGTHS)
    lens = LENGTHS + [0]
    k, v, q = _rows(10, B, L, heads, dh, dtype), _rows(11, B, L, heads, dh, dtype), _rows(12, B, n, H, dh, dtype, spread=0.2)
    ctx = _ctx(H, dh, dtype)
    kv = _empty_cache(B, heads, L + 3, dh, fill=255, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    kk, vv = _load(kv, k, v)
    for b, length in enumerate(lens):                         # what lies behind a sample's rows is NaN
        kv.k_scale[b, :, length:] = 255
        kv.v_scale[b, :, length:] = 255
    o = _attend(ctx, to_dev(q, dtype), kv, dtype, B, n)
    want = kvq.attention(q, kk, vv, dh ** -0.5, lens)
    assert not to_np(o[-1]).any()
    for b in range(B):
        assert np.isfinite(to_np(o[b])).all(), lens[b]
    _check(f"lengths {dtype} {dh} {H}/{heads} n {n}", o, want, dtype)
    for b in range(len(LENGTHS)):                             # each length under its own norm
        _check(f"  length {lens[b]}", o[b], want[b], dtype)


@pytest.mark.parametrize("dtype,dh,H,heads,B,n,L", [
    ("bf16", 128, 16, 16, 1, 1, 5000), ("bf16", 128, 8, 2, 3, 1, 3001), ("bf16", 64, 30, 30, 2, 1, 871), ("bf16", 64, 4, 4, 1, 231, 871),
    ("bf16", 128, 4, 4, 2, 130, 1497), ("bf16", 128, 2, 2, 1, 600, 2000), ("bf16", 64, 2, 1, 1, 300, 700), ("bf16", 64, 4, 2, 9, 129, 65),
    ("bf16", 128, 32, 4, 2, 5, 1100), ("f32", 64, 16, 16, 2, 128, 552), ("f32", 128, 4, 2, 1, 33, 2300), ("f32", 64, 4, 4, 5, 1, 1025)])
def test_attention_at_sizes_of_use(dtype, dh, H, heads, B, n, L):
    k, v, q = _rows(20, B, L, heads, dh, dtype), _rows(21, B, L, heads, dh, dtype), _rows(22, B, n, H, dh, dtype, spread=0.2)
    ctx, kv = _ctx(H, dh, dtype), _empty_cache(B, heads, L, dh, len=L)
    kk, vv = _load(kv, k, v)
    qd = to_dev(q, dtype)
    o = _attend(ctx, qd, kv, dtype, B, n)
    _check(f"{dtype} {dh} {H}/{heads} {B}x{n}x{L}", o, kvq.attention(q, kk, vv, dh ** -0.5, [L] * B), dtype)
    assert torch.equal(o, _attend(ctx, qd, kv, dtype, B, n))   # the same answer again


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh,H,heads,n", [(128, 4, 4, 1), (64, 4, 2, 40), (128, 4, 4, 200), (64, 8, 8, 200)])
def test_attention_with_hidden_rows(dtype, dh, H, heads, n):
    """Masks that leave all, some, one or no row of a sample; what hidden rows hold, NaN too, has no influence."""
    L = 700
    g = np.random.default_rng(30)
    masks = [np.ones(L), g.random(L) < 0.7, g.random(L) < 0.02, np.zeros(L), np.arange(L) == 0, np.arange(L) == L - 1,
             np.arange(L) >= 640, np.arange(L) < 64, (np.arange(L) // 64) % 2, np.arange(L) == 333]
    mask, B = np.array(masks).astype(np.uint8), len(masks)
    mask[1] *= 255                                            # any byte but 0
    k, v, q = _rows(31, B, L, heads, dh, dtype), _rows(32, B, L, heads, dh, dtype), _rows(33, B, n, H, dh, dtype, spread=0.2)
    ctx = _ctx(H, dh, dtype)
    kv = _empty_cache(B, heads, L, dh, len=L, mask=torch.from_numpy(mask).cuda())
    kk, vv = _load(kv, k, v)
    hidden = torch.from_numpy(mask == 0).cuda()[:, None, :, None]
    for t in (kv.k_scale, kv.v_scale):
        t.masked_fill_(hidden, 255)
    o = _attend(ctx, to_dev(q, dtype), kv, dtype, B, n)
    want = kvq.attention(q, kk, vv, dh ** -0.5, [L] * B, mask)
    assert not to_np(o[3]).any()
    for b in range(B):
        _check(f"mask {b} {dtype} {dh} n {n}", o[b], want[b], dtype)
    for b, t in ((4, 0), (5, L - 1), (9, 333)):               # one visible row: its values, rounded to nothing (they are exact)
        assert np.array_equal(to_np(o[b]), np.repeat(vv[b, None, :, t], H // heads, axis=1).repeat(n, 0).astype(np.float32))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh,n", [(128, 2), (64, 150), (128, 150)])
def test_attention_passes_on_what_is_not_a_number(dtype, dh, n):
    """A NaN in a visible value, key or query makes exactly the outputs NaN that it takes part in."""
    H, heads, L, B = 2, 1, 300, 5
    k, v, q = _rows(40, B, L, heads, dh, dtype), _rows(41, B, L, heads, dh, dtype), _rows(42, B, n, H, dh, dtype)
    ctx, kv = _ctx(H, dh, dtype), _empty_cache(B, heads, L, dh, len=L)
    kk, vv = _load(kv, k, v)
    kv.v_scale[1, 0, 70, 1] = 255                             # one block of one row's values
    kv.k_scale[2, 0, 299, 0] = 255                            # ... of one key
    qd = to_dev(q, dtype)
    qd[3, n - 1, 1, 5], qd[4, 0, 0, dh - 1] = float("nan"), float("inf")
    o = to_np(_attend(ctx, qd, kv, dtype, B, n))
    want = kvq.attention(q, kk, vv, dh ** -0.5, [L] * B)
    bad = np.zeros(o.shape, bool)
    bad[1, :, :, 32:64], bad[2], bad[3, n - 1, 1], bad[4, 0, 0] = True, True, True, True
    assert np.array_equal(np.isnan(o), bad)
    _check(f"beside NaN {dtype} {dh} {n}", torch.from_numpy(np.where(bad, 0, o)), np.where(bad, 0, want), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh,n", [(128, 1), (64, 33), (128, 140), (64, 140)])
@pytest.mark.parametrize("case", ["sharp", "rising", "falling", "tiny values", "huge values", "mixed values", "tiny queries", "huge queries", "huge keys"])
def test_attention_over_the_range_of_scores_and_values(dtype, dh, n, case):
    """Running maxima that move at every row, values and queries of every size that the format holds."""
    H, heads, L, B = 2, 2, 421, 2
    k, v, q = _rows(50, B, L, heads, dh, dtype), _rows(51, B, L, heads, dh, dtype), _rows(52, B, n, H, dh, dtype, spread=0.2)
    up = 2.0 ** np.linspace(-10, 4, L).astype(np.float32)[None, :, None, None]
    if case == "sharp":
        q = q * 8
    elif case in ("rising", "falling"):                       # scores grow or shrink along the rows, by 2^14 in all
        q, k = np.abs(q), np.abs(k) * (up if case == "rising" else up[:, ::-1])
    elif case == "tiny values":
        v = v * np.float32(2.0 ** -110)
    elif case == "huge values":
        v = v * np.float32(2.0 ** 115)
    elif case == "mixed values":                              # sizes from 2^-30 to 1, in no order
        v = v * 2.0 ** -np.random.default_rng(53).integers(0, 31, (B, L, heads, 1)).astype(np.float32)
    elif case == "tiny queries":
        q = q * np.float32(2.0 ** -100)
    elif case == "huge queries":                              # with small keys: the scores are of use
        q, k = q * np.float32(2.0 ** 80), k * np.float32(2.0 ** -80)
    elif case == "huge keys":
        q, k = q * np.float32(2.0 ** -90), k * np.float32(2.0 ** 90)
    if dtype == "bf16":
        q, k, v = wl.round_to_bf16(q), wl.round_to_bf16(k), wl.round_to_bf16(v)
    ctx, kv = _ctx(H, dh, dtype), _empty_cache(B, heads, L, dh, len=L)
    kk, vv = _load(kv, k, v)
    o = _attend(ctx, to_dev(q, dtype), kv, dtype, B, n)
    want = kvq.attention(q, kk, vv, dh ** -0.5, [L] * B)
    if case in ("rising", "falling", "sharp"):
        # scores up to s carry a relative error of one rounding of the query (2^-9 bf16, 2^-23 fp32) times s into the weights:
        # held to twice that times the spread of the values
        s = dh ** -0.5 * np.einsum("bnhd,bhtd->bhnt", np.abs(q).astype(np.float64), np.abs(kk))
        rel = np.minimum(2 * s.max() * (2.0 ** -9 if dtype == "bf16" else 2.0 ** -22), 2.0)
        lim = rel * np.abs(vv).max() + (2.0 ** -8 if dtype == "bf16" else 1e-5) * np.abs(want)
        assert (np.abs(to_np(o) - want) <= lim + 1e-6).all()
        assert np.isfinite(to_np(o)).all()
        return
    scale = np.abs(want).max()                                # so that squares stay in range
    got = to_np(o).astype(np.float64) / scale
    _check(f"{case} {dtype} {dh} {n}", torch.from_numpy(got), want / scale, dtype)


def test_attention_of_equal_scores_is_the_mean():
    """Queries of 0: every visible row weighs the same, and only sum and output are rounded."""
    for dtype, dh, n, L in (("bf16", 128, 3, 1000), ("bf16", 64, 200, 777), ("bf16", 128, 200, 777), ("f32", 64, 20, 777)):
        H = heads = 2
        v = _rows(60, 1, L, heads, dh, dtype)
        ctx, kv = _ctx(H, dh, dtype), _empty_cache(1, heads, L, dh, len=L)
        _, vv = _load(kv, _rows(61, 1, L, heads, dh, dtype), v)
        o = to_np(_attend(ctx, torch.zeros((1, n, H, dh), dtype=tdtype(dtype), device="cuda"), kv, dtype, 1, n))
        want = vv.mean(2)[:, None]
        # fp32 sum of L terms (L * 2^-24 of their mean size) and the output's rounding
        lim = (2.0 ** -8 if dtype == "bf16" else 2.0 ** -23) * np.abs(want) + L * 2.0 ** -24 * np.abs(vv).mean(2)[:, None]
        assert (np.abs(o - want) <= lim).all()


@pytest.mark.parametrize("dtype,dh,n", [("bf16", 64, 600), ("bf16", 128, 600), ("bf16", 128, 20), ("f32", 64, 20)])
def test_queries_half_way_between_numbers_of_few_bits(dtype, dh, n):
    """Queries whose elements, in units of log2, lie half-way between two numbers with three bits of mantissa, over one key, and on such
    numbers over another, of the same score: what is left of the queries, added over a row, must not show in the weights."""
    B, H, L, quarter = 8, 8, 440, dh // 4
    ctx = _ctx(H, dh, dtype, attn_scale=float(np.log(2)))
    sign = np.random.default_rng(20).choice([-1.0, 1.0], dh)
    ties = [4.25, 4.75, 5.25, 5.75, 6.25, 6.75, 7.25]
    q, k, v = np.zeros((B, n, H, dh), np.float32), np.zeros((B, L, H, dh), np.float32), _rows(21, B, L, H, dh, dtype)
    for r in range(n):
        t = ties[r % len(ties)]
        q[:, r] = np.repeat([t, t, 4.0, t - 4.0], quarter) * sign
    k[:, 3, :, :quarter] = sign[:quarter]                    # scores of quarter * t, both
    k[:, 300, :, 2 * quarter:] = sign[2 * quarter:]
    kv = _empty_cache(B, H, L, dh, len=L)
    kk, vv = _load(kv, k, v)
    _check(f"half-way {dtype} {dh} n {n}", _attend(ctx, to_dev(q, dtype), kv, dtype, B, n),
           kvq.attention(q, kk, vv, np.log(2), [L] * B), dtype)


def test_attention_scale_of_the_context():
    H, dh, n, L = 2, 64, 5, 90
    k, v, q = _rows(70, 1, L, H, dh, "f32"), _rows(71, 1, L, H, dh, "f32"), _rows(72, 1, n, H, dh, "f32")
    ctx, kv = _ctx(H, dh, "f32", attn_scale=0.3), _empty_cache(1, H, L, dh, len=L)
    kk, vv = _load(kv, k, v)
    _check("scale", _attend(ctx, to_dev(q, "f32"), kv, "f32", 1, n), kvq.attention(q, kk, vv, 0.3, [L]), "f32")


@pytest.mark.parametrize("n", [1, 130])
def test_offsets_beyond_32_bits(n):
    """The last sample of a cache of 5.4 GB per tensor: appended, read back and attended over."""
    B, H, dh, cap, rows = 40, 16, 128, 131072, 77
    ctx = _ctx(H, dh, "bf16")
    e = lambda last: torch.empty((B, H, cap, last), dtype=torch.uint8, device="cuda")
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    lens[-1] = cap - rows
    kv = fv.KVQ(e(64), e(64), e(4), e(4), lens=lens, mask=torch.zeros((B, cap), dtype=torch.uint8, device="cuda"))
    kv.mask[-1, cap - rows:] = 1
    x = _rows(80, 1, rows, 2 * H, dh, "bf16")
    k, v = x[:, :, :H], x[:, :, H:]
    kd, vd = torch.zeros((B, rows, H, dh), dtype=torch.bfloat16, device="cuda"), torch.zeros((B, rows, H, dh), dtype=torch.bfloat16, device="cuda")
    kd[-1:], vd[-1:] = to_dev(k, "bf16"), to_dev(v, "bf16")
    fv.fvar_kvq_append(ctx, kv, kd, vd, B, rows)
    lens += rows
    kb, vb = torch.empty_like(kd), torch.empty_like(vd)
    fv.fvar_kvq_read(ctx, kv, B, -rows, rows, kb, vb)
    held = [kvq.values(*kvq.quantise(np.swapaxes(t, 1, 2))) for t in (k, v)]
    assert np.array_equal(to_np(kb[-1:]), held[0].swapaxes(1, 2).astype(np.float32))
    assert np.array_equal(to_np(vb[-1:]), held[1].swapaxes(1, 2).astype(np.float32))
    q = _rows(81, 1, n, H, dh, "bf16", spread=0.2)
    qd = torch.zeros((B, n, H, dh), dtype=torch.bfloat16, device="cuda")
    qd[-1:] = to_dev(q, "bf16")
    o = _attend(ctx, qd, kv, "bf16", B, n)
    assert not o[:-1].any()
    _check(f"far {n}", o[-1:], kvq.attention(q, *held, dh ** -0.5, [rows]), "bf16")


@pytest.mark.parametrize("dtype,n,L", [("bf16", 1, 2000), ("bf16", 150, 900), ("f32", 3, 500)])
def test_calls_in_a_captured_graph(dtype, n, L):
    """Append and attention as nodes of a graph, replayed with new rows and lengths between other work."""
    B, H, heads, dh, new = 2, 4, 2, 128, n
    ctx = _ctx(H, dh, dtype)
    lens, total = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    kv = _empty_cache(B, heads, L + 4 * new, dh, lens=lens)
    after = fv.KVQ(kv.k, kv.v, kv.k_scale, kv.v_scale, lens=total)
    _load(kv, _rows(90, B, L, heads, dh, dtype), _rows(91, B, L, heads, dh, dtype))
    kd, vd, qd = (torch.zeros((B, new, m, dh), dtype=tdtype(dtype), device="cuda") for m in (heads, heads, H))
    o = torch.empty((B, n, H, dh), dtype=tdtype(dtype), device="cuda")
    ws = torch.empty(fv.fvar_kvq_attention_workspace_bytes(ctx, after, B, n), dtype=torch.uint8, device="cuda")

    def step():
        fv.fvar_kvq_append(ctx, kv, kd, vd, B, new)
        fv.fvar_kvq_attention(ctx, qd, after, B, n, o, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for r in range(3):
        lens.copy_(torch.tensor([L + r * new, L // 2 + r * new], dtype=torch.int32))
        total.copy_(lens + new)
        for i, t in enumerate((kd, vd, qd)):
            t.copy_(to_dev(_rows(92 + 3 * r + i, B, new, t.shape[2], dh, dtype), dtype))
        o.fill_(float("nan"))
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        got = o.clone()
        held = [kvq.values(c.cpu().numpy(), s.cpu().numpy()) for c, s in ((kv.k, kv.k_scale), (kv.v, kv.v_scale))]
        for b in range(B):                                    # the rows just written are the oracle's
            at = int(lens[b])
            c, _ = kvq.quantise(np.swapaxes(to_np(kd), 1, 2))
            assert np.array_equal(kv.k[b, :, at:at + new].cpu().numpy(), c[b])
        _check(f"graph {dtype} replay {r}", got, kvq.attention(to_np(qd), *held, dh ** -0.5, total.cpu().tolist()), dtype)
        o.fill_(float("nan"))
        step()
        torch.cuda.synchronize()
        assert torch.equal(o, got)


def test_lengths_are_checked_when_asked():
    ctx, lens = _ctx(2, 64, "bf16"), torch.tensor([3, 7], dtype=torch.int32, device="cuda")
    kv = _empty_cache(2, 2, 10, 64, lens=lens)
    x, q = torch.zeros((2, 4, 2, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 1, 2, 64), dtype=torch.bfloat16, device="cuda")
    fv.fvar_kvq_append(ctx, kv, x, x, 2, 4)                   # unchecked: what does not fit is left out
    fv.fvar_debug_checks(ctx, True)
    with pytest.raises(fv.FvarError, match="lens"):
        fv.fvar_kvq_append(ctx, kv, x, x, 2, 4)
    fv.fvar_kvq_append(ctx, kv, x[:, :3].contiguous(), x[:, :3].contiguous(), 2, 3)
    _attend(ctx, q, kv, "bf16", 2, 1)
    lens[0] = -1
    with pytest.raises(fv.FvarError, match="lens"):
        _attend(ctx, q, kv, "bf16", 2, 1)
    with pytest.raises(fv.FvarError, match="lens"):
        fv.fvar_kvq_read(ctx, kv, 2, 0, 1, k=q)


# ------------------------------------------------------------------------------------ the block
@pytest.mark.parametrize("dtype,d,H,B,M,keep,Lp,ragged", [
    ("bf16", 256, 4, 2, 40, 40, 100, False), ("bf16", 512, 4, 1, 300, 90, 333, False), ("bf16", 128, 2, 3, 17, 1, 50, True), ("f32", 256, 4, 2, 33, 12, 70, True)])
def test_block_over_the_cache(dtype, d, H, B, M, keep, Lp, ragged):
    """The block with W_o = 1 and an MLP of 0 gives x + attention: against the oracle's attention over the cache that the
    block left, whose new rows are the oracle's quantisation of the plain block's K and V rows, bit for bit."""
    dh, F = d // H, 64
    x = wl.activations_lowrank(B, M, d, seed=100 + M, bf16=dtype == "bf16")
    g = np.random.default_rng(101)
    bf = lambda a: wl.round_to_bf16(a) if dtype == "bf16" else a.astype(np.float32)
    w = {"w_qkv": bf(0.05 * g.standard_normal((3 * d, d))), "b_qkv": bf(0.1 * g.standard_normal(3 * d)), "w_o": np.eye(d, dtype=np.float32),
         "w_fc1": np.zeros((F, d), np.float32), "w_fc2": np.zeros((d, F), np.float32)}
    wd = {n: to_dev(a, dtype) for n, a in w.items()}
    turned = dict(wd, w_qkv=wd["w_qkv"].roll(d, 0).contiguous(), b_qkv=wd["b_qkv"].roll(d, 0).contiguous())   # q rows come out as K rows
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
        return to_np(K[:, Lp:Lp + keep]), to_np(V[:, Lp:Lp + keep])

    (kn, vn), (qn, _) = plain(wd), plain(turned)
    lens = [Lp - 9 * b for b in range(B)] if ragged else [Lp] * B
    kv = _empty_cache(B, H, cap, dh, len=Lp, lens=torch.tensor(lens, dtype=torch.int32, device="cuda") if ragged else None)
    _load(kv, _rows(102, B, Lp, H, dh, dtype), _rows(103, B, Lp, H, dh, dtype))
    size = fv.fvar_block_kvq_workspace_bytes(ctx, kv, B, keep)
    ws, y = torch.full((size,), 255, dtype=torch.uint8, device="cuda"), torch.empty((B, keep, d), dtype=tdtype(dtype), device="cuda")
    fv.fvar_debug_checks(ctx, True)                           # with the canary behind the workspace
    size = fv.fvar_block_kvq_workspace_bytes(ctx, kv, B, keep)
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    if keep == M:
        fv.fvar_block_forward_dense_kvq(ctx, wd, xd, B, M, kv, y, ws)
    else:
        fv.fvar_block_forward_pruned_kvq(ctx, wd, xd, B, M, idx_d, keep, kv, y, ws)
    fv.fvar_debug_checks(ctx, False)
    for rows, codes, scales in ((kn, kv.k, kv.k_scale), (vn, kv.v, kv.v_scale)):
        c, s = kvq.quantise(np.swapaxes(rows, 1, 2))
        for b in range(B):
            assert np.array_equal(codes[b, :, lens[b]:lens[b] + keep].cpu().numpy(), c[b])
            assert np.array_equal(scales[b, :, lens[b]:lens[b] + keep].cpu().numpy(), s[b])
    held = [kvq.values(c.cpu().numpy(), s.cpu().numpy()) for c, s in ((kv.k, kv.k_scale), (kv.v, kv.v_scale))]
    att = kvq.attention(qn, *held, dh ** -0.5, [n + keep for n in lens]).reshape(B, keep, d)
    xk = np.stack([x[b, idx[b]] for b in range(B)])
    _check(f"block {dtype} {B}x{keep}", y, xk + att, dtype)


def test_example_of_scales_over_the_cache():
    """The example's chain: the 4-bit cache changes a scale's output by the error of the values it holds, about a tenth of the attention's
    part of a row whose residual it is added to."""
    import workloads
    from examples.kvq_scales import run

    W = workloads.Workload("small", 256, 4, 64, 512, (1, 2, 4, 9, 12), (9, 12), 2, 5, 16, 2, 2, "bf16")
    lines = []
    far = run(W, W.scales, 2, 2, out=lines.append)
    assert sorted(far) == [1, 2, 4, 9, 12] and all(0 < x < 0.1 for x in far.values()), far
    assert len(lines) == 7 and "read back" in lines[-1]


@pytest.mark.parametrize("dtype,n", [("bf16", 1), ("bf16", 140), ("f32", 3)])
def test_lengths_outside_the_cache_are_held_to_it(dtype, n):
    B, H, dh, cap = 4, 2, 64, 90
    lens = [-7, 2 ** 31 - 1, cap + 1, 40]
    ctx = _ctx(H, dh, dtype)
    kv = _empty_cache(B, H, cap, dh, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    kk, vv = _load(kv, _rows(110, B, cap, H, dh, dtype), _rows(111, B, cap, H, dh, dtype))
    q = _rows(112, B, n, H, dh, dtype, spread=0.2)
    o = _attend(ctx, to_dev(q, dtype), kv, dtype, B, n)
    assert not to_np(o[0]).any()
    _check(f"held to the cache {dtype} {n}", o, kvq.attention(q, kk, vv, dh ** -0.5, [0, cap, cap, 40]), dtype)
