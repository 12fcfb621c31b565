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
