"""Rotary positions on the GPU through the C ABI, against the definition in 64 bits.

fp32: the angle's fraction of a turn is exact to 2^-30, sine and cosine are off by 2 units of 2^-24 at most, and a result has two products and a sum, each
rounded: at most 6 * 2^-24 of (|x| + |y|) * magnitude.  bf16: that, and the result's own rounding, 2^-8 of it at most.  Elements that are
not turned stay as they are, bit for bit."""
import numpy as np
import pytest
import torch

import paper_2512_16483_amd as fv
import workloads as wl
from oracle import rope

pytestmark = pytest.mark.gpu

from gpu_util import tdtype, to_dev, to_np  # noqa: E402


def _ctx(H, dh, dtype):
    return fv.Context(hidden=H * dh, heads=H, head_dim=dh, ffn_hidden=256, dtype=dtype)


def _draw(seed, dtype, *shape):
    x = np.random.default_rng(seed).standard_normal(shape).astype(np.float32)
    return wl.round_to_bf16(x) if dtype == "bf16" else x


def _check(got, x, pos, f, dtype, dim, axes=1, interleaved=False, magnitude=1.0):
    want = rope.rotate(x, pos, f, dim, axes, interleaved, magnitude)
    got, P = to_np(got).astype(np.float64), dim // axes
    part = np.abs(x[..., :dim].astype(np.float64)).reshape(*x.shape[:-1], axes, P)
    pair = part.reshape(*part.shape[:-1], P // 2, 2).sum(-1, keepdims=True) if interleaved else (part[..., :P // 2] + part[..., P // 2:])[..., None]
    size = np.broadcast_to(pair, (*pair.shape[:-1], 2))
    size = size.reshape(part.shape) if interleaved else np.moveaxis(size, -1, -2).reshape(part.shape)
    room = 6 * 2.0 ** -24 * magnitude * size.reshape(*x.shape[:-1], dim)
    if dtype == "bf16":
        room = room * 1.01 + 2.0 ** -8 * np.abs(want[..., :dim])
    off = np.abs(got - want)[..., :dim]
    assert (off <= room).all(), float((off - room).max())
    assert np.array_equal(got[..., dim:], x[..., dim:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,heads,dh,B,n,dim,axes,interleaved", [
    (4, 4, 64, 1, 1, 64, 1, False), (4, 2, 64, 2, 3, 16, 1, True), (30, 30, 64, 2, 17, 32, 2, False), (32, 8, 128, 5, 1, 128, 1, True),
    (16, 16, 128, 1, 33, 128, 2, False), (8, 1, 128, 3, 7, 96, 2, True), (2, 2, 128, 1, 2501, 112, 1, False), (2, 1, 64, 3, 1001, 48, 1, True),
    (3, 3, 64, 1, 2049, 64, 2, True), (1, 1, 128, 2, 1027, 16, 1, False)])
def test_rope_of_packed_rows(dtype, H, heads, dh, B, n, dim, axes, interleaved):
    q, k = _draw(1, dtype, B, n, H, dh), _draw(2, dtype, B, n, heads, dh)
    pos = np.random.default_rng(3).integers(-50, 2000, (B, n, axes)).astype(np.int32)
    ctx, r = _ctx(H, dh, dtype), fv.Rope(dim=dim, axes=axes, interleaved=interleaved)
    out = lambda x: torch.full(x.shape, float("nan"), dtype=tdtype(dtype), device="cuda")
    qd, kd, p = to_dev(q, dtype), to_dev(k, dtype), torch.from_numpy(pos).cuda()
    qo, ko = out(q), out(k)
    fv.fvar_rope_apply(ctx, r, p, B, n, qd, kd, qo, ko)
    f = rope.frequencies(dim // axes)
    _check(qo, q, pos, f, dtype, dim, axes, interleaved)
    _check(ko, k, pos, f, dtype, dim, axes, interleaved)
    assert np.array_equal(to_np(qd), q) and np.array_equal(to_np(kd), k)
    only = out(k)                                             # keys alone, queries alone, in place
    fv.fvar_rope_apply(ctx, r, p, B, n, k=kd, k_out=only)
    assert torch.equal(only, ko)
    fv.fvar_rope_apply(ctx, r, p, B, n, qd)
    assert torch.equal(qd, qo)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kw", [dict(scaling="linear", factor=8.0), dict(scaling="ntk", factor=8.0, base=5e5),
                                dict(scaling="yarn", factor=16.0, original=4096.0, low=1.0, high=32.0, magnitude=1.2773)])
@pytest.mark.parametrize("far", [2 ** 20, 2 ** 30])
def test_rope_far_out_and_scaled(dtype, kw, far):
    H, heads, dh, B, n = 4, 2, 128, 2, 9
    x = _draw(4, dtype, B, n, H + 2 * heads, dh)
    pos = (far + np.arange(B * n).reshape(B, n, 1) * 12345).astype(np.int32)
    fused = to_dev(x, dtype)
    rest = fused[:, :, H + heads:].clone()
    ctx, r = _ctx(H, dh, dtype), fv.Rope(dim=dh, **kw)
    # the queries and keys of a fused projection, in place
    fv.fvar_rope_apply(ctx, r, torch.from_numpy(pos).cuda(), B, n, fused[:, :, :H], fused[:, :, H:H + heads])
    f = np.array(r.turns) * 2 * np.pi                         # (the table itself is held to the oracle's on the host)
    _check(fused[:, :, :H], x[:, :, :H], pos, f, dtype, dh, magnitude=kw.get("magnitude", 1.0))
    _check(fused[:, :, H:H + heads], x[:, :, H:H + heads], pos, f, dtype, dh, magnitude=kw.get("magnitude", 1.0))
    assert torch.equal(fused[:, :, H + heads:], rest)


def test_rope_with_frequencies_of_ones_own_and_rows_apart():
    H, dh, B, n = 2, 64, 1, 5
    x = _draw(5, "f32", B, n, 2 * H, dh)
    xd = to_dev(x, "f32")
    out = torch.full((B, n, 3 * H, dh), -7.0, device="cuda")
    turns = [0.25] * 16
    fv.fvar_rope_apply(_ctx(H, dh, "f32"), fv.Rope(dim=32, turns=turns), torch.arange(n, dtype=torch.int32, device="cuda"), B, n,
                       xd[:, :, H:], q_out=out[:, :, H:2 * H])
    _check(out[:, :, H:2 * H], x[:, :, H:], np.arange(n).reshape(1, n, 1), np.full(16, np.pi / 2), "f32", 32)
    assert (out[:, :, :H] == -7).all() and (out[:, :, 2 * H:] == -7).all()


def test_rope_keeps_what_is_not_finite_to_its_pair():
    H, dh = 1, 64
    x = np.ones((1, 1, H, dh), np.float32)
    x[..., 3], x[..., 40] = np.inf, np.nan
    xd = to_dev(x, "bf16")
    fv.fvar_rope_apply(_ctx(H, dh, "bf16"), fv.Rope(dim=64), torch.tensor([[5]], dtype=torch.int32, device="cuda"), 1, 1, xd)
    bad = ~np.isfinite(to_np(xd))[0, 0, 0]
    assert set(np.flatnonzero(bad)) == {3, 35, 8, 40}


def test_rope_on_another_stream_and_in_a_graph():
    H, dh, B, n = 8, 128, 2, 300
    x = _draw(6, "bf16", B, n, H, dh)
    pos = torch.arange(B * n, dtype=torch.int32, device="cuda")
    ctx, r, xd = _ctx(H, dh, "bf16"), fv.Rope(dim=dh), to_dev(x, "bf16")
    want, out = torch.empty_like(xd), torch.empty_like(xd)
    fv.fvar_rope_apply(ctx, r, pos, B, n, xd, q_out=want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    fv.fvar_rope_apply(ctx, r, pos, B, n, xd, q_out=out, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fv.fvar_rope_apply(ctx, r, pos, B, n, xd, q_out=out)
    for shift in (0, 1, 100):
        pos.copy_(torch.arange(B * n, dtype=torch.int32, device="cuda") + shift)
        fv.fvar_rope_apply(ctx, r, pos, B, n, xd, q_out=want)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_rows_whose_offsets_pass_32_bits():
    H, dh, n = 16, 64, 2_200_001
    q = torch.randn((1, n, H, dh), dtype=torch.bfloat16, device="cuda")
    pos = torch.arange(n, dtype=torch.int32, device="cuda").reshape(1, n, 1)
    out = torch.empty_like(q)
    fv.fvar_rope_apply(_ctx(H, dh, "bf16"), fv.Rope(dim=dh), pos, 1, n, q, None, out)
    at = [0, 1, n // 2, 2 ** 21 - 1, 2 ** 21, n - 2, n - 1]
    _check(out[:, at], to_np(q[:, at]), np.array(at, np.int32).reshape(1, -1, 1), rope.frequencies(dh), "bf16", dh)


def test_a_magnitude_of_0_stands_for_1():
    ctx, r = _ctx(2, 64, "f32"), fv.Rope(dim=64)
    q, pos = torch.randn((1, 5, 2, 64), device="cuda"), torch.arange(5, dtype=torch.int32, device="cuda").reshape(1, 5, 1)
    one, two = torch.empty_like(q), torch.empty_like(q)
    fv.fvar_rope_apply(ctx, r, pos, 1, 5, q, None, one)
    r._c.magnitude = 0.0                                      # as a program with frequencies of its own may leave it
    fv.fvar_rope_apply(ctx, r, pos, 1, 5, q, None, two)
    assert torch.equal(one, two) and not torch.equal(one, q)
