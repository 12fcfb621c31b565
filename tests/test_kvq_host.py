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


def test_sizes_that_the_calls_refuse_need_no_workspace():
    lib = fv.load_library()
    ctx = fv.Context(hidden=256, heads=4, head_dim=64, ffn_hidden=256)
    for fn in (lib.fvar_kvq_attention_workspace_bytes, lib.fvar_block_kvq_workspace_bytes):
        size = lambda B, n, **kw: fn(ctx.handle, C.byref(_cache(kv_heads=4, **kw)), B, n)
        assert size(1, 10, capacity=1 << 24) > 0 and size(1, 10, capacity=(1 << 24) + 1) == 0
        assert size(16384, 1, capacity=1 << 24) == 0                              # B * kv_heads
        assert size(1, (1 << 23) + 1) == 0 and size(1, 2 ** 31 - 1) == 0 and size(2 ** 31 - 1, 2 ** 31 - 1) == 0
        if fn is lib.fvar_block_kvq_workspace_bytes:                              # (the attention by itself may need none)
            assert size(16383, 512) > 0 and size(1, 1 << 23) > 0


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


# ------------------------------------------------------------------------------------ ways of running the attention
def ways(dtype, B, n, H, heads, dh, length, ragged):
    """(rows of a block, wavefronts of its workgroup, shares of the keys of a divided block)"""
    w = fv.load_library()["_ZN4fvar18kvq_attention_waysEiiiiiiii"](dtype == "bf16", B, n, H, heads, dh, length, ragged)
    return w // 100000, w // 1000 % 100, w % 1000


# dtype, head_dim, heads, kv heads, samples, queries, keys, lengths of their own, way
WAYS = {
    "16 rows, 1 wavefront": ("bf16", 64, 16, 16, 32, 40, 100, False, (16, 1, 1)),
    "16 rows, 1 wavefront, 128": ("bf16", 128, 16, 16, 24, 40, 97, False, (16, 1, 1)),
    "16 rows, 1 wavefront, ragged": ("bf16", 128, 16, 16, 24, 40, 128, True, (16, 1, 1)),
    "16 rows, 1 wavefront, fp32": ("f32", 64, 8, 8, 16, 130, 70, False, (16, 1, 1)),
    "16 rows, 2 wavefronts": ("bf16", 128, 16, 16, 16, 40, 300, False, (16, 2, 1)),
    "16 rows, 2 wavefronts, 64": ("bf16", 64, 32, 8, 32, 10, 333, False, (16, 2, 1)),
    "16 rows, 2 wavefronts, fp32": ("f32", 128, 8, 8, 12, 130, 201, False, (16, 2, 1)),
    "16 rows, 4 wavefronts": ("bf16", 128, 8, 8, 16, 40, 600, False, (16, 4, 1)),
    "16 rows, 4 wavefronts, fp32": ("f32", 64, 4, 4, 9, 200, 511, False, (16, 4, 1)),
    "16 rows, 3 shares": ("bf16", 128, 8, 2, 3, 30, 900, False, (16, 4, 3)),
    "16 rows, 20 shares": ("bf16", 64, 4, 4, 1, 3, 5151, False, (16, 4, 20)),
    "16 rows, 20 shares, fp32": ("f32", 128, 4, 4, 1, 3, 5151, False, (16, 4, 20)),
    "16 rows, shares of ragged samples": ("bf16", 128, 8, 8, 32, 1, 2100, True, (16, 4, 2)),
    "128 rows, whole": ("bf16", 128, 8, 8, 32, 200, 330, False, (128, 4, 1)),
    "128 rows, whole, 64": ("bf16", 64, 8, 8, 32, 200, 330, False, (128, 4, 1)),
    "128 rows, two groups": ("bf16", 128, 4, 4, 20, 230, 900, False, (128, 8, 1)),
    "128 rows, two groups, 64": ("bf16", 64, 4, 2, 32, 130, 1000, False, (128, 8, 1)),
    "128 rows, two groups, ragged": ("bf16", 64, 8, 8, 14, 240, 1000, True, (128, 8, 1)),
    "128 rows, two groups, divided": ("bf16", 128, 8, 8, 4, 230, 3600, False, (128, 8, 4)),
    "128 rows, two groups, many shares": ("bf16", 64, 8, 2, 1, 130, 16000, False, (128, 8, 16)),
    "128 rows, two groups, ragged shares": ("bf16", 128, 4, 4, 9, 200, 2300, True, (128, 8, 3)),
    "128 rows, two groups, the rest divided": ("bf16", 128, 11, 11, 12, 200, 2100, False, (128, 8, 4)),
    "128 rows, two groups, the rest divided, ragged": ("bf16", 64, 10, 5, 13, 200, 2050, True, (128, 8, 4)),
    "128 rows, one group, divided": ("bf16", 128, 4, 4, 18, 129, 4100, False, (128, 4, 3)),
    "128 rows, last round divided": ("bf16", 64, 16, 16, 31, 200, 1100, False, (128, 4, 3)),
    "128 rows, last round divided, 128": ("bf16", 128, 4, 4, 70, 200, 600, True, (128, 4, 2)),
    "128 rows, last round divided, ragged": ("bf16", 128, 16, 8, 40, 90, 1400, True, (128, 4, 4)),
}


@pytest.mark.parametrize("case", sorted(WAYS))
def test_ways_that_the_gpu_tests_are_there_for(case):
    """tests/test_gpu_kvq_ways.py runs these: another choice of constants must not take a way out of its reach unseen."""
    dtype, dh, H, heads, B, n, L, ragged, expect = WAYS[case]
    assert ways(dtype, B, n, H, heads, dh, L, ragged) == expect


def test_small_changes_of_length_and_lengths_of_their_own_need_no_more_workspace():
    lib = fv.load_library()
    for dtype in ("bf16", "f32"):
        for heads, kv_heads, dh in ((16, 16, 128), (30, 30, 64), (32, 4, 128)):
            ctx = fv.Context(hidden=heads * dh, heads=heads, head_dim=dh, ffn_hidden=64, dtype=dtype)
            for B in (1, 3, 32):
                for n in (1, 7, 48, 64, 128, 129, 700):
                    last = 0
                    for cap in (1, 100, 127, 128, 400, 1024, 1025, 3000, 12121, 100000):
                        size = lib.fvar_kvq_attention_workspace_bytes(ctx.handle, C.byref(_cache(kv_heads=kv_heads, capacity=cap, len=1)), B, n)
                        assert size >= last                   # never falls as the capacity grows
                        last = size
                        block, _, shares = ways(dtype, B, n, heads, kv_heads, dh, cap, False)
                        units = B * kv_heads * -(-(n * heads // kv_heads) // block)
                        if shares > 1 and units < 256:        # every unit divided
                            assert size >= 4 * units * shares * block * (dh + 2)


def test_workspace_never_falls_where_the_choice_of_groups_changes():
    """What a length takes is in the size of a cache of that capacity; a longer one has to be enough for it, on both sides of every change."""
    lib = fv.load_library()
    caps = [1000, 1500, 2040, 2047, 2048, 2049, 2500, 4000, 4095, 4096, 4097, 5000, 9000]
    for heads, dh in ((16, 128), (30, 64), (8, 64), (12, 128)):
        ctx = fv.Context(hidden=heads * dh, heads=heads, head_dim=dh, ffn_hidden=64, dtype="bf16")
        for B in (1, 3, 8):
            for n in range(100, 4600, 257):
                size = [lib.fvar_kvq_attention_workspace_bytes(ctx.handle, C.byref(_cache(kv_heads=heads, capacity=c, len=1)), B, n) for c in caps]
                assert size == sorted(size), (heads, dh, B, n, size)
