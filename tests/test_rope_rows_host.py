"""Rows that fvar_rope_apply can turn, and those that share memory, without a GPU: refusals come before anything is launched."""
import ctypes as C
import itertools
import math
import random

import pytest
import torch

import paper_2512_16483_amd as fv
from test_kvb_host import _Fake

INV = fv.FVAR_ERR_INVALID_ARG


def _rope(dim=64, axes=1):
    r = fv._Rope(dim=dim, axes=axes, base=1e4, factor=1.0)
    assert fv.load_library().fvar_rope_init(C.byref(r)) == 0
    return r


def _apply(B=1, n=4, kv_heads=4, q=None, ld_q=0, k=None, ld_k=0, q_out=None, ld_q_out=0, k_out=None, ld_k_out=0, pos=0x10, axes=1):
    """The status of a call with 4 heads of 64 in bf16: rows of 512 bytes of queries."""
    ctx = fv.Context(hidden=256, heads=4, head_dim=64, ffn_hidden=256)
    return fv.load_library().fvar_rope_apply(ctx.handle, None, C.byref(_rope(axes=axes)), pos, B, n, kv_heads, q, ld_q, k, ld_k, q_out, ld_q_out,
                                             k_out, ld_k_out)


BASE = 0x100000


def test_outputs_that_share_memory_with_another_tensor_are_refused():
    far = BASE + (1 << 20)
    assert _apply(q=BASE, q_out=BASE + 512) == INV and _apply(q=BASE, q_out=BASE - 512) == INV                 # its own input, by a row
    assert _apply(q=BASE, q_out=BASE + 3 * 512) == INV and _apply(q=BASE, q_out=BASE + 3 * 512 + 496) == INV
    assert _apply(q=BASE, k=far, q_out=far, k_out=BASE) == INV                                                 # one changed for the other
    assert _apply(q=BASE, k=far, q_out=far + 512, k_out=far) == INV
    assert _apply(q=BASE, k=far, q_out=BASE, k_out=BASE + 1024) == INV
    assert _apply(q=BASE, k=BASE, q_out=BASE, k_out=far) == INV                                                # a tensor that is turned in place and read
    assert _apply(q=BASE, k=BASE, q_out=BASE, k_out=BASE) == INV
    assert _apply(q=BASE, k=far, q_out=2 * far, k_out=2 * far + 512) == INV                                    # both outputs
    assert _apply(q=BASE, q_out=far, pos=far + 1024 + 4) == INV and _apply(q=BASE, q_out=far, pos=far + 2048 - 4) == INV
    # rows that lie apart: parts of one tensor that meet
    assert _apply(q=BASE, ld_q=768, q_out=BASE + 496, ld_q_out=768) == INV
    assert _apply(q=BASE, ld_q=768, q_out=BASE + 1536 - 496, ld_q_out=768) == INV
    assert _apply(q=BASE, ld_q=768, q_out=BASE + 1024, ld_q_out=520) == INV                                    # of different distances
    assert _apply(q=BASE, ld_q=768, k=BASE + 496, ld_k=768, q_out=BASE, ld_q_out=768, k_out=BASE + 496, ld_k_out=768) == INV


@pytest.mark.parametrize("seed", range(4))
def test_rows_share_memory_where_bytes_do(seed):
    """Against the sets of bytes themselves, a call's q and q_out."""
    rng, lib = random.Random(seed), fv.load_library()
    share = lib["_ZN4fvar17rows_share_memoryEmlllmlll"]
    share.argtypes, share.restype = [C.c_size_t, C.c_long, C.c_long, C.c_long] * 2, C.c_bool
    for _ in range(3000):
        n, wa, wb = rng.randint(1, 6), rng.randint(1, 5), rng.randint(1, 5)
        m = rng.choice([n, 1])
        la = wa + rng.choice([0, 0, 1, 3, 7])
        lb = rng.choice([la, wb, wb + rng.randint(0, 9)])
        lb = max(lb, wb)
        a, b = 1000, 1000 + rng.randint(-40, 40)
        bytes_of = lambda at, w, ld, rows: set(itertools.chain.from_iterable(range(at + i * ld, at + i * ld + w) for i in range(rows)))
        assert share(a, wa, la, n, b, wb, lb, m) == bool(bytes_of(a, wa, la, n) & bytes_of(b, wb, lb, m)), (a, wa, la, n, b, wb, lb, m)


@pytest.mark.parametrize("name,value", [("turns", math.nan), ("turns", math.inf), ("turns", -math.inf), ("magnitude", 1e39), ("magnitude", -1e300),
                                        ("magnitude", 1e-46)])
@pytest.mark.parametrize("pair", [0, 13, 31])
def test_a_table_that_is_no_number_is_refused(name, value, pair):
    """Frequencies that a program wrote itself; a magnitude that fp32 does not hold, or holds as 0."""
    ctx, lib, r = fv.Context(hidden=256, heads=4, head_dim=64, ffn_hidden=256), fv.load_library(), _rope()
    if name == "turns":
        r.turns[pair] = value
        with pytest.raises(ValueError):
            fv.Rope(dim=64, turns=[value if i == pair else 0.1 for i in range(32)])
    else:
        r.magnitude = value
        with pytest.raises(fv.FvarError):
            fv.Rope(dim=64, magnitude=value)
    assert lib.fvar_rope_apply(ctx.handle, None, C.byref(r), 0x10, 1, 4, 4, BASE, 0, None, 0, BASE, 0, None, 0) == INV
    kv = fv._KVB(0x100000, 0x200000, 0x300000, 0x400000, None, None, 4, 100, 50)
    w = C.byref(fv._Weights(*[0x1000] * 12))
    assert lib.fvar_block_forward_dense_kvb(ctx.handle, None, w, 0x1000, 1, 1, C.byref(kv), C.byref(r), 0x10, None, 0, 0x1000, 0x1000, 1 << 40) == INV
    r = _rope(dim=32)
    r.turns[16] = math.nan                                    # behind the table's pairs: not read
    assert lib.fvar_rope_apply(ctx.handle, None, C.byref(r), 0x10, 1, 4, 4, BASE, 0, None, 0, BASE + 512, 0, None, 0) == INV   # (refused for its rows)
    assert b"shares memory" in lib.fvar_last_error(ctx.handle)


@pytest.mark.parametrize("B,n", [(0, 4), (2, 0), (-1, 4), (2, -3), (0, 0)])
def test_the_binding_refuses_no_rows(B, n):
    bf16, i32 = (lambda *s: _Fake(*s, dtype=torch.bfloat16)), lambda *s: _Fake(*s, dtype=torch.int32)
    ctx, r = fv.Context(hidden=256, heads=4, head_dim=64, ffn_hidden=256), fv.Rope(dim=64)
    for kw in (dict(q=bf16(2, 4, 4, 64)), dict(k=bf16(2, 4, 4, 64)), dict(q=bf16(2, 4, 4, 64), k=bf16(2, 4, 2, 64))):
        with pytest.raises(ValueError):
            fv.fvar_rope_apply(ctx, r, i32(2, 4), B, n, stream=0, **kw)
