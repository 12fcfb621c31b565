"""The 4-bit cache without a GPU: the oracle against the definition element by element, and the refusals of the C ABI and
of the binding, which come before anything is launched."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2512_16483_amd as fv
from oracle import kvq


# ------------------------------------------------------------------------------------ oracle
def test_oracle_rounds_to_the_nearest_value_ties_to_the_even_code():
    mids = [(0.25, 0), (0.75, 2), (1.25, 2), (1.75, 4), (2.5, 4), (3.5, 6), (5.0, 6)]
    x = np.zeros((1, 32))
    x[0, 31] = 6.0                                            # e = 0
    x[0, :7] = [m for m, _ in mids]
    x[0, 7:14] = [-m for m, _ in mids]
    x[0, 14:21] = [np.nextafter(m, 0) for m, _ in mids]
    x[0, 21:28] = [np.nextafter(m, 9) for m, _ in mids]
    codes, scales = kvq.quantise(x)
    c = np.stack([codes & 15, codes >> 4], -1).reshape(-1)
    assert scales.tolist() == [[127]]
    even = [code for _, code in mids]
    assert c[:7].tolist() == even and c[7:14].tolist() == [8 + e for e in even]
    assert c[14:21].tolist() == list(range(7)) and c[21:28].tolist() == list(range(1, 8))


@pytest.mark.parametrize("top,e", [(6.0, 0), (6.999, 0), (7.0, 1), (13.99, 1), (14.0, 2), (3.5, 0), (3.499, -1), (0.0, -124),
                                   (1e-45, -124), (7 * 2.0 ** -124, -123), (3.4028234663852886e38, 125), (1.75 * 2.0 ** 127, 125)])
def test_oracle_takes_the_smallest_scale_that_holds_the_block(top, e):
    x = np.zeros((1, 32))
    x[0, 5] = -top
    codes, scales = kvq.quantise(x)
    assert int(scales[0, 0]) - 127 == e
    assert np.isfinite(kvq.values(codes, scales)).all()


def test_oracle_error_is_at_most_half_a_step_and_what_is_not_finite_stays_so():
    x = np.random.default_rng(1).standard_normal((200, 64)) * np.exp(np.random.default_rng(2).normal(0, 3, (200, 1)))
    codes, scales = kvq.quantise(x)
    y, size = kvq.values(codes, scales), np.repeat(2.0 ** (scales.astype(float) - 127), 32, axis=-1)
    half = np.where(np.abs(x) < 2 * size, 0.25, np.where(np.abs(x) < 4 * size, 0.5, 1.0)) * size
    assert (np.abs(x - y) <= half).all()
    again, same = kvq.quantise(y)                             # what has been held once is held unchanged
    assert np.array_equal(kvq.values(again, same), y)
    for bad in (np.nan, np.inf, -np.inf):
        z = x[:1].copy()
        z[0, 40] = bad
        codes, scales = kvq.quantise(z)
        assert scales[0, 1] == 255 and np.isnan(kvq.values(codes, scales)[0, 32:]).all()
        assert np.isfinite(kvq.values(codes, scales)[0, :32]).all()


def test_oracle_attention_without_a_visible_row_is_zero():
    g = np.random.default_rng(3)
    q, k, v = g.standard_normal((2, 3, 4, 64)), g.standard_normal((2, 2, 5, 64)), g.standard_normal((2, 2, 5, 64))
    mask = np.ones((2, 5))
    mask[1, :2] = 0
    o = kvq.attention(q, k, v, 0.125, [0, 3], mask)
    assert not o[0].any() and np.allclose(o[1], v[1, np.array([0, 0, 1, 1]), 2])


# ------------------------------------------------------------------------------------ refusals
def _cache(**kw):
    a = dict(k=0x1000, v=0x1000, k_scale=0x1000, v_scale=0x1000, lens=None, mask=None, kv_heads=2, capacity=100, len=50)
    a.update(kw)
    return fv._KVQ(*[a[n] for n in ("k", "v", "k_scale", "v_scale", "lens", "mask", "kv_heads", "capacity", "len")])


BAD_CACHES = [(dict(k=None), 1), (dict(v=None), 1), (dict(k_scale=None), 1), (dict(v_scale=None), 1), (dict(k=0x1008), 1),
              (dict(v_scale=0x1004), 1), (dict(lens=0x1002), 1), (dict(kv_heads=0), 1), (dict(kv_heads=3), 1),
              (dict(kv_heads=-2), 1), (dict(capacity=0), 1), (dict(len=-1), 1), (dict(len=101), 1),
              (dict(capacity=(1 << 24) + 1), 2)]


@pytest.mark.parametrize("kw,status", BAD_CACHES)
@pytest.mark.parametrize("name", ["append", "read", "attention", "dense", "pruned"])
def test_calls_refuse_a_cache_that_is_none(name, kw, status):
    lib, fake = fv.load_library(), 0x1000
    ctx = fv.Context(hidden=256, heads=4, head_dim=64, ffn_hidden=256)
    if name in ("dense", "pruned"):
        kw = dict(dict(kv_heads=4), **kw)
    kv, w, h = C.byref(_cache(**kw)), C.byref(fv._Weights(*[fake] * 12)), ctx.handle
    got = {"append": lambda: lib.fvar_kvq_append(h, None, kv, fake, fake, 0, 1, 1),
           "read": lambda: lib.fvar_kvq_read(h, None, kv, 1, 0, 1, fake, fake),
           "attention": lambda: lib.fvar_kvq_attention(h, None, fake, 0, kv, 1, 1, fake, fake, 1 << 40),
           "dense": lambda: lib.fvar_block_forward_dense_kvq(h, None, w, fake, 1, 1, kv, fake, fake, 1 << 40),
           "pruned": lambda: lib.fvar_block_forward_pruned_kvq(h, None, w, fake, 1, 2, fake, 1, kv, fake, fake, 1 << 40)}[name]()
    assert got == status and lib.fvar_last_error(h)


def test_calls_refuse_what_they_cannot_do():
    lib, fake, inv = fv.load_library(), 0x1000, fv.FVAR_ERR_INVALID_ARG
    ctx = fv.Context(hidden=256, heads=4, head_dim=64, ffn_hidden=256)
    h, kv = ctx.handle, C.byref(_cache())
    app = lambda *a: lib.fvar_kvq_append(h, None, *a)
    assert app(None, fake, fake, 0, 1, 1) == inv
    assert app(kv, None, fake, 0, 1, 1) == inv and app(kv, fake, None, 0, 1, 1) == inv
    assert app(kv, fake + 8, fake, 0, 1, 1) == inv
    assert app(kv, fake, fake, 0, 0, 1) == inv and app(kv, fake, fake, 0, 1, 0) == inv
    assert app(kv, fake, fake, 0, 1, 51) == inv                                   # 50 + 51 > 100
    assert app(kv, fake, fake, 120, 1, 1) == inv and app(kv, fake, fake, 132, 1, 1) == inv and app(kv, fake, fake, -8, 1, 1) == inv
    assert app(kv, fake, fake, 0, 32768, 1) == fv.FVAR_ERR_UNSUPPORTED            # B * kv_heads
    rd = lambda *a: lib.fvar_kvq_read(h, None, kv, *a)
    assert rd(1, 0, 1, None, None) == inv and rd(1, 0, 1, fake + 2, None) == inv
    assert rd(0, 0, 1, fake, fake) == inv and rd(1, 0, 0, fake, fake) == inv
    assert rd(1, 50, 51, fake, fake) == inv and rd(1, -101, 1, fake, fake) == inv and rd(1, 0, 101, fake, fake) == inv
    assert rd(1, 2 ** 31 - 1, 1, fake, fake) == inv and rd(1, -2 ** 31, 1, fake, fake) == inv
    att = lambda q, ld, B, n, o, ws=fake, size=1 << 40: lib.fvar_kvq_attention(h, None, q, ld, kv, B, n, o, ws, size)
    assert att(None, 0, 1, 1, fake) == inv and att(fake, 0, 1, 1, None) == inv
    assert att(fake + 4, 0, 1, 1, fake) == inv and att(fake, 0, 1, 1, fake + 4) == inv and att(fake, 0, 1, 1, fake, fake + 4) == inv
    assert att(fake, 0, 1, 0, fake) == inv and att(fake, 0, 0, 1, fake) == inv
    assert att(fake, 248, 1, 1, fake) == inv and att(fake, 260, 1, 1, fake) == inv
    assert att(fake, 0, 1, 1 << 24, fake) == fv.FVAR_ERR_UNSUPPORTED
    assert lib.fvar_kvq_append(None, None, kv, fake, fake, 0, 1, 1) == inv and lib.fvar_kvq_read(None, None, kv, 1, 0, 1, fake, fake) == inv
    assert lib.fvar_kvq_attention(None, None, fake, 0, kv, 1, 1, fake, fake, 1) == inv
    # the block: kv heads of its own number, workspace
    w, kv4 = C.byref(fv._Weights(*[fake] * 12)), C.byref(_cache(kv_heads=4))
    blk = lambda cache, M, size: lib.fvar_block_forward_dense_kvq(h, None, w, fake, 1, M, cache, fake, fake, size)
    assert blk(kv, 10, 1 << 40) == fv.FVAR_ERR_UNSUPPORTED and b"kv_heads" in lib.fvar_last_error(h)
    assert blk(kv4, 51, 1 << 40) == inv and blk(None, 10, 1 << 40) == inv
    need = lib.fvar_block_kvq_workspace_bytes(h, kv4, 1, 10)
    assert need > 0 and blk(kv4, 10, need - 1) == fv.FVAR_ERR_WORKSPACE
    assert lib.fvar_block_forward_pruned_kvq(h, None, w, fake, 1, 20, None, 10, kv4, fake, fake, need) == inv


def test_workspace_sizes_do_not_read_the_pointers():
    lib = fv.load_library()
    ctx = fv.Context(hidden=256, heads=4, head_dim=64, ffn_hidden=256)
    h = ctx.handle
    empty = _cache(k=None, v=None, k_scale=None, v_scale=None)
    for fn in (lib.fvar_kvq_attention_workspace_bytes, lib.fvar_block_kvq_workspace_bytes):
        assert fn(h, C.byref(empty), 1, 10) == fn(h, C.byref(_cache()), 1, 10) and fn(h, C.byref(empty), 1, 10) % 256 == 0
        assert fn(h, None, 1, 10) == 0 and fn(None, C.byref(empty), 1, 10) == 0
        assert fn(h, C.byref(empty), 0, 10) == 0 and fn(h, C.byref(empty), 1, 0) == 0
        assert fn(h, C.byref(_cache(kv_heads=3)), 1, 10) == 0
    # the block's own workspace holds the new rows on their way into the cache
    assert lib.fvar_block_kvq_workspace_bytes(h, C.byref(_cache(kv_heads=4)), 2, 30) >= lib.fvar_block_workspace_bytes(h, 2, 30)


def test_binding_refuses_tensors_that_do_not_fit():
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)
    good = dict(k=u8(2, 4, 10, 32), v=u8(2, 4, 10, 32), k_scale=u8(2, 4, 10, 2), v_scale=u8(2, 4, 10, 2))
    for kw in (dict(v=u8(2, 4, 9, 32)), dict(k_scale=u8(2, 4, 10, 1)), dict(lens=torch.zeros(3, dtype=torch.int32)),
               dict(lens=torch.zeros(2, dtype=torch.int64)), dict(mask=u8(2, 9)), dict(mask=torch.zeros(2, 10)),
               dict(v=good["v"].float())):
        with pytest.raises(ValueError):
            fv.KVQ(**dict(good, **kw))
    with pytest.raises(ValueError, match="GPU"):
        fv.KVQ(**good)                                        # right shapes, but host memory
