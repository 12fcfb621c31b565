"""The 8-bit cache, its eviction and rotary positions without a GPU: the oracles against their definitions, and the refusals of the C ABI and
of the binding, which come before anything is launched."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2512_16483_amd as fv
from oracle import kvb, rope


# ------------------------------------------------------------------------------------ oracles
def test_oracle_values_are_those_of_the_library_type():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    got = kvb.values(codes.numpy().reshape(1, 256), np.array([127], np.uint8))[0]
    assert np.array_equal(got, want, equal_nan=True)


def test_oracle_rounds_to_the_nearest_value_ties_to_the_even_code():
    mids = kvb.MIDS
    even = [i if i % 2 == 0 else i + 1 for i in range(126)]
    assert kvb.encode(mids, 0).tolist() == even and kvb.encode(-mids, 0).tolist() == [128 + c for c in even]
    assert kvb.encode(np.nextafter(mids, 0), 0).tolist() == list(range(126))
    assert kvb.encode(np.nextafter(mids, 999), 0).tolist() == list(range(1, 127))
    assert kvb.encode(np.array([464.0, 448.0, 449.0, 0.0, -0.0, np.inf, -np.inf, np.nan]), 0).tolist() == [126, 126, 126, 0, 128, 127, 127, 127]
    x = np.random.default_rng(1).standard_normal(4000).astype(np.float32) * 50
    assert np.array_equal(kvb.encode(x, 0), torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


@pytest.mark.parametrize("top,e", [(464.0, 0), (464.001, 1), (448.0, 0), (232.0, -1), (232.0001, 0), (0.0, -117), (1e-45, -117),
                                   (464 * 2.0 ** 118, 118), (464 * 2.0 ** 118 * 1.01, 119), (3.4028234663852886e38, 119)])
def test_oracle_takes_the_smallest_power_that_serves(top, e):
    assert int(kvb.least(np.array(top))) == e
    assert np.isfinite(kvb.VALUES[126] * 2.0 ** e) and (e == 119 or top == 0 or kvb.VALUES[126] * 2.0 ** e >= top * 0.965)


def test_oracle_append_raises_a_blocks_power_and_rounds_what_it_holds():
    codes, scales = np.full((1, 1, 40, 64), 0x55, np.uint8), np.full((1, 1, 2), 0x55, np.uint8)
    x = np.full((1, 3, 1, 64), 1.125)
    kvb.append(codes, scales, [30], x[:, :1])                 # the block holds 0x55 rows of power 0x55 - 127
    assert scales[0, 0, 0] == int(kvb.least(np.array(1.125))) + 127 and scales[0, 0, 1] == 0x55
    assert not kvb.values(codes, scales)[0, 0, :30].any()     # 2^-42 of the new row's size
    kvb.append(codes, scales, [31], 4 * x)
    assert (kvb.values(codes, scales)[0, 0, 30] == 1.125).all() and (kvb.values(codes, scales)[0, 0, 31] == 4.5).all()
    assert (kvb.values(codes, scales)[0, 0, 32:34] == 4.5).all() and (codes[0, 0, 34:] == 0x55).all()
    kvb.append(codes, scales, [34], 1e-3 * x)                 # a smaller row does not lower it
    assert scales[0, 0, 1] == int(kvb.least(np.array(4.5))) + 127


def test_oracle_eviction_by_hand():
    codes, scales = np.zeros((2, 1, 8, 64), np.uint8), np.full((2, 1, 1), 127, np.uint8)
    codes[...] = (np.arange(8) + 8)[None, None, :, None]
    w = np.zeros((2, 1, 8))
    w[0, 0] = [3, 1, 3, 2, 3, 0, np.nan, 9]
    w[1, 0] = [0, 0, 0, 0, 0, 0, 0, 0]
    mask = np.ones((2, 8), np.uint8)
    mask[1, [1, 2, 3, 4, 5, 6]] = 0
    idx, counts, out = kvb.evict(codes, scales, w, [7, 8], 4, 1, mask)
    assert idx[0, 0].tolist() == [0, 2, 4, 6] and counts.tolist() == [4, 2] and idx[1, 0].tolist() == [0, 7, -1, -1]
    assert np.array_equal(kvb.values(*out[0][0])[:, 0], kvb.VALUES[[8, 10, 12, 14]])
    assert kvb.evict(codes, scales, w, [7, 8], 3, 0)[0][0, 0].tolist() == [0, 2, 6]      # not a number before all numbers, ties to the lowest


def test_oracle_attention_weights_sum_to_the_rows_of_queries():
    g = np.random.default_rng(3)
    q, k, v = g.standard_normal((2, 3, 4, 64)), g.standard_normal((2, 2, 5, 64)), g.standard_normal((2, 2, 5, 64))
    mask = np.ones((2, 5))
    mask[1, :2] = 0
    o, w = kvb.attention(q, k, v, 0.125, [0, 3], mask)
    assert not o[0].any() and not w[0].any() and np.allclose(o[1], v[1, np.array([0, 0, 1, 1]), 2])
    assert np.allclose(w[1, :, 2], 6) and not w[1, :, [0, 1, 3, 4]].any()


@pytest.mark.parametrize("kw", [{}, dict(scaling="linear", factor=4.0), dict(scaling="ntk", factor=8.0),
                                dict(scaling="yarn", factor=8.0, original=4096.0, low=1.0, high=32.0)])
@pytest.mark.parametrize("dim,axes", [(16, 1), (64, 1), (64, 2), (128, 1), (128, 2), (96, 2)])
def test_rope_table_is_the_oracles(kw, dim, axes):
    r = fv.Rope(dim=dim, axes=axes, base=5e5, **kw)
    want = rope.frequencies(dim // axes, base=5e5, **kw)
    assert np.allclose(np.array(r.turns) * 2 * math.pi, want, rtol=1e-13, atol=0)
    assert r._c.magnitude == 1.0 and fv.Rope(dim=16, magnitude=0.5)._c.magnitude == 0.5


def test_oracle_rope_keeps_scores_of_equal_distances():
    g = np.random.default_rng(2)
    x, y = g.standard_normal((1, 1, 1, 64)), g.standard_normal((1, 1, 1, 64))
    f = rope.frequencies(64)
    at = lambda z, p, **kw: rope.rotate(z, np.full((1, 1, 1), p), f, 64, **kw)
    for kw in ({}, dict(interleaved=True)):
        one = (at(x, 7, **kw) * at(y, 3, **kw)).sum()
        assert np.isclose(one, (at(x, 1004, **kw) * at(y, 1000, **kw)).sum()) and np.allclose(at(x, 0, **kw), x)
    grid = rope.rotate(x, np.array([[[3, 5]]]), rope.frequencies(16), 32, axes=2)
    assert np.array_equal(grid[..., 32:], x[..., 32:])
    assert np.allclose(grid[..., :16], rope.rotate(x[..., :16], np.full((1, 1, 1), 3), rope.frequencies(16), 16))
    assert np.allclose(grid[..., 16:32], rope.rotate(x[..., 16:32], np.full((1, 1, 1), 5), rope.frequencies(16), 16))


# ------------------------------------------------------------------------------------ refusals
def _cache(**kw):
    a = dict(k=0x100000, v=0x200000, k_scale=0x300001, v_scale=0x400003, lens=None, mask=None, kv_heads=2, capacity=100, len=50)
    a.update(kw)
    return fv._KVB(*[a[n] for n in ("k", "v", "k_scale", "v_scale", "lens", "mask", "kv_heads", "capacity", "len")])


BAD_CACHES = [(dict(k=None), 1), (dict(v=None), 1), (dict(k_scale=None), 1), (dict(v_scale=None), 1), (dict(k=0x1008), 1),
              (dict(v=0x1004), 1), (dict(lens=0x1002), 1), (dict(kv_heads=0), 1), (dict(kv_heads=3), 1),
              (dict(kv_heads=-2), 1), (dict(capacity=0), 1), (dict(len=-1), 1), (dict(len=101), 1),
              (dict(capacity=(1 << 24) + 1), 2)]


@pytest.mark.parametrize("kw,status", BAD_CACHES)
@pytest.mark.parametrize("name", ["append", "read", "attention", "evict", "dense", "pruned"])
def test_calls_refuse_a_cache_that_is_none(name, kw, status):
    lib, fake = fv.load_library(), 0x1000
    ctx = fv.Context(hidden=256, heads=4, head_dim=64, ffn_hidden=256)
    if name in ("dense", "pruned"):
        kw = dict(dict(kv_heads=4), **kw)
    w = C.byref(fv._Weights(*[fake] * 12))
    kv, h, to = C.byref(_cache(**kw)), ctx.handle, C.byref(_cache(k=0x500000, v=0x600000, k_scale=0x700000, v_scale=0x800000))
    got = {"append": lambda: lib.fvar_kvb_append(h, None, kv, fake, fake, 0, 1, 1),
           "read": lambda: lib.fvar_kvb_read(h, None, kv, 1, 0, 1, fake, fake),
           "attention": lambda: lib.fvar_kvb_attention(h, None, fake, 0, kv, 1, 1, fake, None, 0, fake, 1 << 40),
           "evict": lambda: lib.fvar_kvb_evict(h, None, kv, fake, 1, 4, 0, to, 0x900000, None, None, fake, 1 << 40),
           "dense": lambda: lib.fvar_block_forward_dense_kvb(h, None, w, fake, 1, 1, kv, None, None, None, 0, fake, fake, 1 << 40),
           "pruned": lambda: lib.fvar_block_forward_pruned_kvb(h, None, w, fake, 1, 2, fake, 1, kv, None, None, None, 0, fake, fake, 1 << 40)}[name]()
    assert got == status and lib.fvar_last_error(h)


def test_calls_refuse_what_they_cannot_do():
    lib, fake, inv, uns = fv.load_library(), 0x1000, fv.FVAR_ERR_INVALID_ARG, fv.FVAR_ERR_UNSUPPORTED
    ctx = fv.Context(hidden=256, heads=4, head_dim=64, ffn_hidden=256)
    h, kv = ctx.handle, C.byref(_cache())
    app = lambda *a: lib.fvar_kvb_append(h, None, *a)
    assert app(None, fake, fake, 0, 1, 1) == inv
    assert app(kv, None, fake, 0, 1, 1) == inv and app(kv, fake, None, 0, 1, 1) == inv and app(kv, fake + 8, fake, 0, 1, 1) == inv
    assert app(kv, fake, fake, 0, 0, 1) == inv and app(kv, fake, fake, 0, 1, 0) == inv and app(kv, fake, fake, 0, 1, 51) == inv
    assert app(kv, fake, fake, 120, 1, 1) == inv and app(kv, fake, fake, 132, 1, 1) == inv and app(kv, fake, fake, -8, 1, 1) == inv
    assert app(kv, fake, fake, 0, 32768, 1) == uns                                # B * kv_heads
    rd = lambda *a: lib.fvar_kvb_read(h, None, kv, *a)
    assert rd(1, 0, 1, None, None) == inv and rd(1, 0, 1, fake + 2, None) == inv
    assert rd(0, 0, 1, fake, fake) == inv and rd(1, 0, 0, fake, fake) == inv
    assert rd(1, 50, 51, fake, fake) == inv and rd(1, -101, 1, fake, fake) == inv and rd(1, 0, 101, fake, fake) == inv
    assert rd(1, 2 ** 31 - 1, 1, fake, fake) == inv and rd(1, -2 ** 31, 1, fake, fake) == inv
    att = lambda q, ld, B, n, o, w=None, ws=fake, size=1 << 40: lib.fvar_kvb_attention(h, None, q, ld, kv, B, n, o, w, 0, ws, size)
    assert att(None, 0, 1, 1, fake) == inv and att(fake, 0, 1, 1, None) == inv
    assert att(fake + 4, 0, 1, 1, fake) == inv and att(fake, 0, 1, 1, fake + 4) == inv and att(fake, 0, 1, 1, fake, None, fake + 4) == inv
    assert att(fake, 0, 1, 1, fake, fake + 4) == inv
    assert att(fake, 0, 1, 0, fake) == inv and att(fake, 0, 0, 1, fake) == inv
    assert att(fake, 248, 1, 1, fake) == inv and att(fake, 260, 1, 1, fake) == inv
    assert att(fake, 0, 1, 1 << 24, fake) == uns
    need = lib.fvar_kvb_attention_workspace_bytes(h, kv, 1, 3, 1)
    assert need > 0 and att(fake, 0, 1, 3, fake, fake, fake, need - 1) == fv.FVAR_ERR_WORKSPACE
    assert att(fake, 0, 1, 3, fake, fake, None, need) == fv.FVAR_ERR_WORKSPACE
    assert lib.fvar_kvb_append(None, None, kv, fake, fake, 0, 1, 1) == inv and lib.fvar_kvb_read(None, None, kv, 1, 0, 1, fake, fake) == inv
    assert lib.fvar_kvb_attention(None, None, fake, 0, kv, 1, 1, fake, None, 0, fake, 1) == inv
    for B, n, kw in ((0, 1, {}), (1, 0, {}), (-1, 1, {}), (1, 1 << 24, {}), (1, 1, dict(kv_heads=3)), (1, 1, dict(capacity=0))):
        assert lib.fvar_kvb_attention_workspace_bytes(h, C.byref(_cache(**kw)), B, n, 1) == 0


def test_eviction_refuses_what_it_cannot_do():
    lib, fake, inv = fv.load_library(), 0x1000, fv.FVAR_ERR_INVALID_ARG
    ctx = fv.Context(hidden=256, heads=4, head_dim=64, ffn_hidden=256)
    h, kv = ctx.handle, C.byref(_cache())
    other = dict(k=0x500000, v=0x600000, k_scale=0x700000, v_scale=0x800000)

    def evict(w=0xa00000, B=1, keep=4, recent=2, to=None, tw=0x900000, lens=None, idx=None, ws=fake, size=1 << 40):
        return lib.fvar_kvb_evict(h, None, kv, w, B, keep, recent, C.byref(_cache(**(other if to is None else to))), tw, lens, idx, ws, size)

    assert evict(w=None) == inv and evict(tw=None) == inv and evict(w=0xa00004) == inv and evict(tw=0x900004) == inv
    assert evict(lens=0x1002) == inv and evict(idx=0x1001) == inv and evict(ws=fake + 4) == inv
    assert evict(keep=0) == inv and evict(recent=-1) == inv and evict(recent=5) == inv and evict(keep=101) == inv
    assert evict(to=dict(other, capacity=3)) == inv and evict(to=dict(other, kv_heads=4)) == inv and evict(to=dict(other, k=None)) == inv
    assert evict(to=dict(other, v_scale=None)) == inv and evict(to=dict(other, k=0x500008)) == inv
    assert evict(to=dict(other, capacity=(1 << 24) + 1)) == fv.FVAR_ERR_UNSUPPORTED
    # one cache in part, caches that share memory, weights that do
    assert evict(to=dict(v=0x600000)) == inv and evict(to=dict(capacity=99)) == inv and evict(to=dict(k_scale=0x700000)) == inv
    assert evict(to=dict(other, k=0x100000 + 64 * 100)) == inv and evict(to=dict(other, v=0x100000 - 64)) == inv
    assert evict(to=dict(other, k_scale=0x200010)) == inv
    assert evict(tw=0xa00000) == inv and evict(to={}, tw=0xa00000 + 16) == inv
    need = lib.fvar_kvb_evict_workspace_bytes(h, kv, 1, 4)
    assert need > 0 and evict(size=need - 1) == fv.FVAR_ERR_WORKSPACE and evict(ws=None) == fv.FVAR_ERR_WORKSPACE
    assert lib.fvar_kvb_evict(None, None, kv, fake, 1, 4, 0, kv, fake, None, None, fake, 1 << 40) == inv
    assert lib.fvar_kvb_evict(h, None, kv, fake, 1, 4, 0, None, fake, None, None, fake, 1 << 40) == inv
    assert lib.fvar_kvb_evict_workspace_bytes(h, kv, 0, 4) == 0 and lib.fvar_kvb_evict_workspace_bytes(h, kv, 1, 0) == 0


def _rope(**kw):
    a = dict(dim=64, axes=1, interleaved=0, scaling=0, base=1e4, factor=2.0, original=100.0, low=1.0, high=32.0, magnitude=0.0)
    a.update(kw)
    return fv._Rope(*[a[n] for n in ("dim", "axes", "interleaved", "scaling", "base", "factor", "original", "low", "high", "magnitude")])


@pytest.mark.parametrize("kw", [dict(dim=0), dict(dim=8), dict(dim=24), dict(dim=144), dict(axes=0), dict(axes=3), dict(dim=48, axes=2),
                                dict(scaling=4), dict(scaling=-1), dict(base=1.0), dict(base=0.0), dict(base=float("nan")),
                                dict(base=float("inf")), dict(scaling=1, factor=0.5), dict(scaling=2, factor=float("nan")),
                                dict(scaling=3, original=0.0), dict(scaling=3, low=32.0), dict(scaling=3, high=float("inf")),
                                dict(magnitude=float("inf"))])
def test_rope_refuses_settings_that_are_none(kw):
    assert fv.load_library().fvar_rope_init(C.byref(_rope(**kw))) == fv.FVAR_ERR_INVALID_ARG
    assert fv.load_library().fvar_rope_init(None) == fv.FVAR_ERR_INVALID_ARG


def test_rope_refuses_rows_that_are_none():
    lib, fake, inv = fv.load_library(), 0x1000, fv.FVAR_ERR_INVALID_ARG
    ctx = fv.Context(hidden=256, heads=4, head_dim=64, ffn_hidden=256)
    h, good = ctx.handle, _rope()
    assert lib.fvar_rope_init(C.byref(good)) == 0

    def apply(r=good, pos=fake, B=1, n=1, kv_heads=2, q=fake, ld_q=0, k=fake, ld_k=0, q_out=fake, ld_q_out=0, k_out=fake, ld_k_out=0):
        return lib.fvar_rope_apply(h, None, None if r is None else C.byref(r), pos, B, n, kv_heads, q, ld_q, k, ld_k, q_out, ld_q_out, k_out, ld_k_out)

    assert apply(r=None) == inv and apply(pos=None) == inv and apply(pos=0x1002) == inv and apply(B=0) == inv and apply(n=0) == inv
    assert apply(r=_rope(dim=128)) == inv and apply(r=_rope(dim=20)) == inv and apply(r=_rope(axes=4)) == inv
    assert apply(q=None, k=None, q_out=None, k_out=None) == inv and apply(q=None) == inv and apply(k_out=None) == inv
    assert apply(kv_heads=0) == inv and apply(kv_heads=3) == inv
    assert apply(q=0x1008) == inv and apply(k_out=0x1004) == inv
    assert apply(ld_q=248) == inv and apply(ld_k=129, ld_k_out=129) == inv and apply(ld_q=264) == inv and apply(ld_q_out=-8) == inv
    assert apply(n=(1 << 24) + 1) == fv.FVAR_ERR_UNSUPPORTED
    assert apply(r=_rope()) == inv                            # never filled in
    odd = _rope()
    lib.fvar_rope_init(C.byref(odd))
    odd.magnitude = float("nan")
    assert apply(r=odd) == inv
    assert lib.fvar_rope_apply(None, None, C.byref(good), fake, 1, 1, 2, fake, 0, None, 0, fake, 0, None, 0) == inv


def test_block_refuses_what_it_cannot_do():
    lib, fake, inv = fv.load_library(), 0x1000, fv.FVAR_ERR_INVALID_ARG
    ctx = fv.Context(hidden=256, heads=4, head_dim=64, ffn_hidden=256)
    h, w, kv, r = ctx.handle, C.byref(fv._Weights(*[fake] * 12)), _cache(kv_heads=4), _rope()
    assert lib.fvar_rope_init(C.byref(r)) == 0

    def dense(kv=kv, rope=r, pos=fake, weights=None, ws=fake, size=1 << 40, M=2):
        return lib.fvar_block_forward_dense_kvb(h, None, w, fake, 1, M, C.byref(kv), None if rope is None else C.byref(rope), pos, weights, 0, fake, ws, size)

    assert dense(kv=_cache(kv_heads=2)) == fv.FVAR_ERR_UNSUPPORTED and dense(M=51) == inv
    assert dense(pos=None) == inv and dense(pos=0x1001) == inv and dense(rope=_rope(dim=128)) == inv and dense(rope=_rope(axes=3)) == inv
    assert dense(rope=None) == inv                            # positions without rope
    assert dense(weights=fake + 8) == inv
    for weigh in (0, 1):
        need = lib.fvar_block_kvb_workspace_bytes(h, C.byref(kv), 1, 2, weigh)
        assert need > 0 and dense(weights=fake if weigh else None, size=need - 1) == fv.FVAR_ERR_WORKSPACE
    assert dense(ws=None) == fv.FVAR_ERR_WORKSPACE
    assert lib.fvar_block_kvb_workspace_bytes(h, C.byref(_cache(kv_heads=3)), 1, 2, 0) == 0
    assert lib.fvar_block_forward_dense_kvb(None, None, w, fake, 1, 1, C.byref(kv), None, None, None, 0, fake, fake, 1 << 40) == inv
    assert lib.fvar_block_forward_dense_kvb(h, None, w, fake, 1, 1, None, None, None, None, 0, fake, fake, 1 << 40) == inv


# ------------------------------------------------------------------------------------ binding
class _Fake:
    """A tensor as the binding looks at one."""

    def __init__(self, *shape, dtype=torch.uint8, strides=None):
        self.t = torch.empty(shape, dtype=dtype)
        self.shape, self.dtype, self.is_cuda = self.t.shape, dtype, True

    def is_contiguous(self):
        return True

    def numel(self):
        return self.t.numel()

    def element_size(self):
        return self.t.element_size()

    def data_ptr(self):
        return 0x1000


def _kvb(B=2, heads=2, cap=40, dh=64, **kw):
    f = lambda *s: _Fake(*s)
    return fv.KVB(f(B, heads, cap, dh), f(B, heads, cap, dh), f(B, heads, (cap + 31) // 32), f(B, heads, (cap + 31) // 32), **kw)


def test_binding_holds_a_cache_to_its_shapes():
    kv = _kvb(len=7)
    assert (kv.batch, kv.kv_heads, kv.capacity, kv.head_dim, kv.len) == (2, 2, 40, 64, 7)
    for name, bad in (("k", _Fake(2, 2, 40, 32)), ("v", _Fake(2, 2, 41, 64)), ("k_scale", _Fake(2, 2, 40, 2)), ("v_scale", _Fake(2, 2, 1)),
                      ("lens", _Fake(2)), ("lens", _Fake(3, dtype=torch.int32)), ("mask", _Fake(2, 39)), ("mask", _Fake(2, 40, dtype=torch.int32)),
                      ("k", None), ("k", _Fake(2, 2, 40, 64, dtype=torch.int8))):
        with pytest.raises(ValueError):
            setattr(kv, name, bad)
    kv.mask = _Fake(2, 40, dtype=torch.bool)
    kv.lens = _Fake(2, dtype=torch.int32)
    ctx = fv.Context(hidden=256, heads=4, head_dim=64, ffn_hidden=256)
    with pytest.raises(ValueError):
        fv.fvar_kvb_attention_workspace_bytes(ctx, kv, 3, 1)
    with pytest.raises(ValueError):
        fv.fvar_kvb_attention_workspace_bytes(fv.Context(hidden=256, heads=2, head_dim=128, ffn_hidden=256), kv, 1, 1)
    bf16 = lambda *s: _Fake(*s, dtype=torch.bfloat16)
    f32 = lambda *s: _Fake(*s, dtype=torch.float32)
    with pytest.raises(ValueError):                           # weights of a wrong type, of a wrong size
        fv.fvar_kvb_attention(ctx, bf16(2, 1, 4, 64), kv, 2, 1, bf16(2, 1, 4, 64), None, weights=bf16(2, 2, 40), stream=0)
    with pytest.raises(ValueError):
        fv.fvar_kvb_attention(ctx, bf16(2, 1, 4, 64), kv, 2, 1, bf16(2, 1, 4, 64), None, weights=f32(2, 2, 39), stream=0)
    with pytest.raises(ValueError):
        fv.fvar_kvb_evict(ctx, kv, f32(2, 2, 40), 2, 8, 0, _kvb(cap=8), f32(2, 2, 40), stream=0)
    with pytest.raises(ValueError):
        fv.fvar_kvb_evict(ctx, kv, f32(2, 2, 40), 2, 8, 0, _kvb(cap=8), f32(2, 2, 8), idx=_Fake(2, 2, 8, dtype=torch.int64), stream=0)
    with pytest.raises(ValueError):
        fv.fvar_rope_apply(ctx, fv.Rope(dim=64, axes=2), _Fake(2, 3, dtype=torch.int32), 2, 3, bf16(2, 3, 4, 64), stream=0)
    with pytest.raises(ValueError):
        fv.Rope(dim=64, turns=[0.1] * 31)
    with pytest.raises(fv.FvarError):
        fv.Rope(dim=40)
    assert fv.Rope(dim=64, turns=[0.25] * 32).turns == [0.25] * 32


def ways(dtype, B, n, H, heads, dh, length, ragged):
    """(rows of a block, wavefronts of a workgroup, shares of a divided block) of an attention."""
    x = fv.load_library()["_ZN4fvar18kvb_attention_waysEiiiiiiii"](dtype == "bf16", B, n, H, heads, dh, length, ragged)
    return x // 100000, x // 1000 % 100, x % 1000


@pytest.mark.parametrize("dtype,B,n,H,heads,dh,length,ragged,expect", [
    ("bf16", 2, 1, 2, 2, 64, 64, 0, (16, 2, 1)), ("bf16", 2, 33, 4, 1, 128, 32, 0, (16, 1, 1)), ("bf16", 32, 64, 16, 16, 128, 150, 0, (16, 1, 1)),
    ("bf16", 16, 64, 16, 16, 64, 500, 1, (16, 2, 1)), ("f32", 40, 60, 16, 16, 64, 90, 0, (16, 1, 1)), ("f32", 16, 70, 16, 16, 64, 200, 0, (16, 2, 1)),
    ("bf16", 2, 7, 30, 30, 64, 100, 0, (16, 4, 1)), ("bf16", 8, 400, 16, 16, 128, 60, 0, (16, 1, 1)),
    ("bf16", 1, 1, 16, 16, 64, 700, 0, (16, 8, 1)), ("bf16", 1, 1, 16, 16, 128, 1300, 0, (16, 8, 2)),
    ("bf16", 2, 3, 16, 4, 128, 9000, 1, (16, 4, 35)), ("bf16", 3, 1, 32, 8, 128, 517, 1, (16, 4, 2)), ("f32", 1, 5, 4, 2, 64, 3000, 0, (16, 8, 5)),
    ("bf16", 3, 257, 4, 4, 64, 700, 0, (16, 8, 1)), ("bf16", 32, 200, 30, 30, 64, 70, 0, (128, 4, 1)), ("bf16", 33, 129, 16, 16, 128, 1030, 0, (128, 4, 4)),
    ("bf16", 4, 512, 16, 16, 64, 4500, 0, (128, 8, 1)), ("bf16", 1, 1000, 2, 1, 128, 6000, 0, (128, 8, 11)), ("bf16", 2, 600, 8, 8, 64, 1700, 0, (128, 8, 3)),
    ("bf16", 5, 230, 16, 16, 64, 4100, 0, (128, 4, 3)), ("bf16", 40, 40, 16, 4, 64, 900, 1, (128, 4, 1))])
def test_sizes_are_run_as_the_gpu_tests_want_them(dtype, B, n, H, heads, dh, length, ragged, expect):
    assert ways(dtype, B, n, H, heads, dh, length, ragged) == expect


def test_no_length_takes_more_workspace_than_the_capacity_is_told():
    lib, g = fv.load_library(), np.random.default_rng(5)
    takes = lib["_ZN4fvar19kvb_attention_takesEiiiiiiiii"]
    takes.restype = C.c_long
    for _ in range(4000):
        dh, group, heads = int(g.choice([64, 128])), int(g.choice([1, 1, 2, 3, 8])), int(np.exp(g.uniform(0, np.log(32))))
        H, B, n = heads * group, int(np.exp(g.uniform(0, np.log(64)))), int(np.exp(g.uniform(0, np.log(3000))))
        cap = int(np.exp(g.uniform(0, np.log(40000))))
        dtype, weights = ("bf16", "f32")[int(g.integers(2))], int(g.integers(2))
        ctx = fv.Context(hidden=H * dh, heads=H, head_dim=dh, ffn_hidden=64, dtype=dtype) if H * dh <= 4096 else None
        if ctx is None:
            continue
        kv = fv._KVB(0x1000, 0x1000, 0x1000, 0x1000, None, None, heads, cap, 0)
        room = lib.fvar_kvb_attention_workspace_bytes(ctx.handle, C.byref(kv), B, n, weights)
        for length in {cap, 1, max(1, cap // 2), max(1, cap // 7), min(cap, 2047), min(cap, 2048), min(cap, 4095), min(cap, 4096), int(g.integers(0, cap + 1))}:
            for ragged in (0, 1):
                assert 4 * takes(dtype == "bf16", B, n, H, heads, dh, length, ragged, weights) <= room, (dtype, B, n, H, heads, dh, length, cap, ragged)


def test_attention_workspace_serves_every_length_and_falls_never_short():
    """What a shorter cache takes is within what the call is told for the capacity."""
    ctx = fv.Context(hidden=256, heads=4, head_dim=64, ffn_hidden=256)
    small = fv.fvar_kvb_attention_workspace_bytes(ctx, _kvb(cap=64), 1, 1)
    assert fv.fvar_kvb_attention_workspace_bytes(ctx, _kvb(cap=64), 1, 1, weights=True) >= small + 8 * 4
    assert fv.fvar_kvb_evict_workspace_bytes(ctx, _kvb(cap=64), 2, 33) >= 2 * 2 * 33 * 4 + 8
