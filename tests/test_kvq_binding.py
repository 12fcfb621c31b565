"""What the binding of the 4-bit cache's calls makes of tensors, without a GPU: host tensors that say of themselves that they are on one,
and a library that notes what it is called with."""
import ctypes as C

import pytest
import torch

import paper_2512_16483_amd as fv


class OnGpu(torch.Tensor):
    is_cuda = property(lambda self: True)


def gpu(t):
    return t.as_subclass(OnGpu)


def zeros(*shape, dtype=torch.bfloat16):
    return gpu(torch.zeros(shape, dtype=dtype))


class Noted:
    """A library whose calls succeed and leave their arguments in `calls`."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 0
        return call


@pytest.fixture
def ctx():
    c = fv.Context(hidden=256, heads=4, head_dim=64, ffn_hidden=256)
    c.real, c.lib = c.lib, Noted()
    yield c
    c.lib = c.real


def cache(B=2, heads=4, capacity=10, **kw):
    u8 = lambda last: zeros(B, heads, capacity, last, dtype=torch.uint8)
    return fv.KVQ(u8(32), u8(32), u8(2), u8(2), **kw)


# ------------------------------------------------------------------------------------ distances between rows
def broadcast():
    """Rows that share memory: one for all samples, one for all rows, and fewer elements apart than a row has."""
    yield zeros(1, 1, 4, 64).expand(2, 1, 4, 64), 2, 1
    yield zeros(1, 1, 4, 64).expand(1, 5, 4, 64), 1, 5
    yield zeros(1, 1, 4, 64).expand(2, 5, 4, 64), 2, 5
    yield zeros(1, 5, 4, 64).expand(2, 5, 4, 64), 2, 5
    yield gpu(torch.zeros(2000, dtype=torch.bfloat16).as_strided((1, 5, 4, 64), (0, 128, 64, 1))), 1, 5


@pytest.mark.parametrize("case", range(5))
def test_rows_that_share_memory_are_refused(ctx, case):
    """A distance of 0 between rows is not one that the calls can be given: for them it stands for packed rows."""
    t, B, n = list(broadcast())[case]
    packed = zeros(B, n, 4, 64)
    with pytest.raises(ValueError):
        fv.fvar_kvq_attention(ctx, t, cache(B), B, n, zeros(B, n, 4, 64), stream=1)
    for k, v in ((t, packed), (packed, t), (t, t)):
        with pytest.raises(ValueError):
            fv.fvar_kvq_append(ctx, cache(B), k, v, B, n, stream=1)
    assert not ctx.lib.calls


def test_rows_apart_are_passed_with_their_distance(ctx):
    qkv = zeros(2, 5, 3 * 256)
    q, k, v = qkv[..., :256], qkv[..., 256:512], qkv[..., 512:]
    fv.fvar_kvq_attention(ctx, q, cache(), 2, 5, zeros(2, 5, 4, 64), stream=1)
    fv.fvar_kvq_append(ctx, cache(), k, v, 2, 5, stream=1)
    fv.fvar_kvq_append(ctx, cache(), k[:, :1], v[:, :1], 2, 1, stream=1)      # one row of each sample: these are five rows apart
    fv.fvar_kvq_append(ctx, cache(), zeros(2, 5, 4, 64), zeros(2, 5, 4, 64), 2, 5, stream=1)
    assert [a[3] for n, a in ctx.lib.calls if n == "fvar_kvq_attention"] == [768]
    assert [a[5] for n, a in ctx.lib.calls if n == "fvar_kvq_append"] == [768, 5 * 768, 0]
    assert ctx.lib.calls[1][1][3] == k.data_ptr() and ctx.lib.calls[1][1][4] == v.data_ptr()


# ------------------------------------------------------------------------------------ types and sizes
def calls(ctx, **kw):
    """Each call that takes rows, with 2 samples and 5 rows (of 6 in the block), one tensor replaced: {name: call}"""
    t = dict(k=zeros(2, 5, 4, 64), v=zeros(2, 5, 4, 64), q=zeros(2, 5, 256), o=zeros(2, 5, 256), x=zeros(2, 6, 256), y=zeros(2, 5, 256),
             y6=zeros(2, 6, 256), keep=zeros(2, 5, dtype=torch.int32))
    t.update(kw)
    ws = zeros(8, dtype=torch.uint8)
    return {"append": lambda: fv.fvar_kvq_append(ctx, cache(), t["k"], t["v"], 2, 5, stream=1),
            "read": lambda: fv.fvar_kvq_read(ctx, cache(), 2, 0, 5, t["k"], t["v"], stream=1),
            "attention": lambda: fv.fvar_kvq_attention(ctx, t["q"], cache(), 2, 5, t["o"], stream=1),
            "dense": lambda: fv.fvar_block_forward_dense_kvq(ctx, {}, t["x"], 2, 6, cache(), t["y6"], ws, stream=1),
            "pruned": lambda: fv.fvar_block_forward_pruned_kvq(ctx, {}, t["x"], 2, 6, t["keep"], 5, cache(), t["y"], ws, stream=1)}


TAKEN = {"append": "kv", "read": "kv", "attention": "qo", "dense": ["x", "y6"], "pruned": ["x", "y", "keep"]}


def test_rows_of_the_right_type_and_size_are_taken(ctx):
    for call in calls(ctx).values():
        call()
    assert len(ctx.lib.calls) == 5
    fv.fvar_kvq_read(ctx, cache(), 2, 0, 5, k=zeros(2, 5, 4, 64), stream=1)
    fv.fvar_kvq_read(ctx, cache(), 2, 0, 5, v=zeros(2 * 5 * 256), stream=1)
    fv.fvar_block_forward_pruned_kvq(ctx, {}, zeros(2, 5, 256), 2, 5, None, 5, cache(), zeros(2, 5, 256), zeros(8, dtype=torch.uint8), stream=1)
    assert len(ctx.lib.calls) == 8


@pytest.mark.parametrize("name,which", [(n, w) for n, ws in TAKEN.items() for w in ws])
def test_rows_of_another_type_are_refused(ctx, name, which):
    """Elements of another size would be read and written past a tensor's end."""
    good = calls(ctx)
    rows = {"x": 6, "y6": 6}.get(which, 5)
    for dtype in (torch.float32, torch.float16, torch.int64, torch.uint8):
        with pytest.raises(ValueError):
            calls(ctx, **{which: zeros(2, rows, 256 if which != "keep" else 1, dtype=dtype)})[name]()
    assert not ctx.lib.calls and name in good


@pytest.mark.parametrize("name,which", [(n, w) for n, ws in TAKEN.items() for w in ws])
def test_rows_too_few_are_refused(ctx, name, which):
    rows, width = {"x": 6, "y6": 6}.get(which, 5), 1 if which == "keep" else 256
    dtype = torch.int32 if which == "keep" else torch.bfloat16
    for shape in ((2, rows - 1, width), (1, rows, width), (2 * rows * width - 1,)):
        with pytest.raises(ValueError):
            calls(ctx, **{which: zeros(*shape, dtype=dtype)})[name]()
    assert not ctx.lib.calls


def test_an_fp32_context_takes_fp32_rows():
    ctx = fv.Context(hidden=256, heads=4, head_dim=64, ffn_hidden=256, dtype="f32")
    real, ctx.lib = ctx.lib, Noted()
    f32 = lambda: zeros(2, 5, 256, dtype=torch.float32)
    fv.fvar_kvq_attention(ctx, f32(), cache(), 2, 5, f32(), stream=1)
    for q, o in ((zeros(2, 5, 256), f32()), (f32(), zeros(2, 5, 256))):
        with pytest.raises(ValueError):
            fv.fvar_kvq_attention(ctx, q, cache(), 2, 5, o, stream=1)
    assert len(ctx.lib.calls) == 1
    ctx.lib = real


def test_room_for_more_rows_is_taken_only_where_the_rows_are_where_the_calls_look(ctx):
    """The first rows of one sample, or of the first samples, are packed; some rows of each of several samples are not."""
    att = lambda q, o, B, n: fv.fvar_kvq_attention(ctx, q, cache(), B, n, o, stream=1)
    more, flat = zeros(2, 9, 4, 64), zeros(5000)
    att(more, more, 1, 5)
    att(more, flat, 1, 9)
    att(zeros(3, 5, 256), zeros(3, 5, 4, 64), 2, 5)
    att(flat, zeros(20, 256), 2, 5)
    att(zeros(10, 4, 64), zeros(1, 10, 256), 2, 5)            # as many elements as are wanted
    assert len(ctx.lib.calls) == 5
    good = zeros(2, 5, 256)
    for bad in (more, zeros(3, 9, 256), zeros(5, 2, 512), zeros(2, 5, 512), zeros(2, 2560)):
        for q, o in ((bad, good), (good, bad)):
            with pytest.raises(ValueError):
                att(q, o, 2, 5)
    with pytest.raises(ValueError):
        att(more, good, 1, 15)                                # rows of one sample and the next
    assert len(ctx.lib.calls) == 5
    pruned = lambda keep, B: fv.fvar_block_forward_pruned_kvq(ctx, {}, zeros(B, 6, 256), B, 6, keep, 5, cache(), zeros(B, 5, 256),
                                                              zeros(8, dtype=torch.uint8), stream=1)
    idx = lambda *s: zeros(*s, dtype=torch.int32)
    for keep, B in ((idx(1, 6), 1), (idx(3, 5), 2), (idx(12), 2)):
        pruned(keep, B)
    with pytest.raises(ValueError):
        pruned(idx(2, 6), 2)
    assert len(ctx.lib.calls) == 8


# ------------------------------------------------------------------------------------ the cache's tensors
@pytest.mark.parametrize("name,shape,dtype", [
    ("k", (2, 4, 10, 32), torch.uint8), ("v", (2, 4, 10, 32), torch.uint8), ("k_scale", (2, 4, 10, 2), torch.uint8),
    ("v_scale", (2, 4, 10, 2), torch.uint8), ("lens", (2,), torch.int32), ("mask", (2, 10), torch.uint8), ("mask", (2, 10), torch.bool)])
def test_a_tensor_assigned_to_a_cache_is_the_one_that_the_calls_read(ctx, name, shape, dtype):
    """Neither the tensor of before, which its caller may have let go, nor one that does not fit."""
    for kv in (cache(), cache(lens=zeros(2, dtype=torch.int32), mask=zeros(2, 10, dtype=torch.uint8))):
        new = zeros(*shape, dtype=dtype)
        setattr(kv, name, new)
        assert getattr(kv, name) is new and getattr(kv._c, name) == new.data_ptr()
        fv.fvar_kvq_append(ctx, kv, zeros(2, 5, 256), zeros(2, 5, 256), 2, 5, stream=1)
        passed = C.cast(ctx.lib.calls[-1][1][2], C.POINTER(fv._KVQ)).contents
        assert getattr(passed, name) == new.data_ptr()
        for bad in (zeros(*shape, dtype=torch.float32), zeros(*shape[:-1], shape[-1] + 1, dtype=dtype), torch.zeros(shape, dtype=dtype),
                    zeros(*shape, 2, dtype=dtype)[..., 0]):
            with pytest.raises(ValueError):
                setattr(kv, name, bad)
            assert getattr(kv, name) is new and getattr(kv._c, name) == new.data_ptr()


def test_lengths_and_masks_come_and_go():
    kv = cache(len=3)
    lens, mask = zeros(2, dtype=torch.int32), zeros(2, 10, dtype=torch.bool)
    kv.lens, kv.mask = lens, mask
    kv.lens = kv.lens + 1                                     # another tensor
    assert kv._c.lens == kv.lens.data_ptr() != lens.data_ptr() and kv._c.mask == mask.data_ptr()
    at = kv.lens
    kv.lens += 1                                              # the same one
    assert kv.lens is at and kv._c.lens == at.data_ptr() and at.tolist() == [2, 2]
    kv.lens = kv.mask = None
    assert kv._c.lens is None and kv._c.mask is None and kv.len == kv._c.len == 3
    for name in ("k", "v", "k_scale", "v_scale"):
        with pytest.raises(ValueError):
            setattr(kv, name, None)
    for name in ("kv_heads", "capacity", "batch", "head_dim"):
        with pytest.raises(AttributeError):
            setattr(kv, name, 1)
