"""Attention over the 4-bit cache in each way in which it is run: blocks of 16 rows by 1, 2 and 4 wavefronts, whole and with the keys divided
between workgroups (few shares and many); blocks of 128 rows, whole, all divided, and with the last round divided; and calls of several
lengths with one workspace.  Bounds: see test_gpu_kvq.py."""
import numpy as np
import pytest
import torch

import paper_2512_16483_amd as fv
from oracle import kvq

pytestmark = pytest.mark.gpu

from gpu_util import to_dev, to_np  # noqa: E402
from test_gpu_kvq import _attend, _check, _ctx, _empty_cache, _load, _rows  # noqa: E402
from test_kvq_host import WAYS, ways  # noqa: E402


@pytest.mark.parametrize("case", sorted(WAYS))
def test_attention_in_every_way(case):
    dtype, dh, H, heads, B, n, L, ragged, expect = WAYS[case]
    assert ways(dtype, B, n, H, heads, dh, L, ragged) == expect
    k, v, q = _rows(1, B, L, heads, dh, dtype), _rows(2, B, L, heads, dh, dtype), _rows(3, B, n, H, dh, dtype, spread=0.2)
    lens = [(L * (b + 1) // B + 7 * b) % (L + 1) if ragged else L for b in range(B)]
    ctx = _ctx(H, dh, dtype)
    kv = _empty_cache(B, heads, L, dh, len=L, lens=torch.tensor(lens, dtype=torch.int32, device="cuda") if ragged else None)
    kk, vv = _load(kv, k, v)
    qd = to_dev(q, dtype)
    o = _attend(ctx, qd, kv, dtype, B, n)
    _check(case, o, kvq.attention(q, kk, vv, dh ** -0.5, lens), dtype)
    assert torch.equal(o, _attend(ctx, qd, kv, dtype, B, n))


@pytest.mark.parametrize("case", sorted(WAYS))
def test_hidden_rows_in_every_way(case):
    """A third of the rows hidden, a stretch of 70, the first and the last of all samples but one, whose rows are all hidden; what they
    hold is not a number."""
    dtype, dh, H, heads, B, n, L, ragged, expect = WAYS[case]
    if n * B * heads * L > 5e7:
        n = max(1, int(5e7 / (B * heads * L)))               # (the same blocks and waves, or others: all are run somewhere)
    g = np.random.default_rng(4)
    k, v, q = _rows(1, B, L, heads, dh, dtype), _rows(2, B, L, heads, dh, dtype), _rows(3, B, n, H, dh, dtype, spread=0.2)
    lens = [(L * (b + 1) // B + 7 * b) % (L + 1) if ragged else L for b in range(B)]
    mask = (g.random((B, L)) < 0.67).astype(np.uint8)
    mask[:, L // 3:L // 3 + 70] = 0
    mask[:, 0] = mask[:, -1] = 0
    if B > 1:
        mask[B // 2] = 0
    kv = _empty_cache(B, heads, L, dh, len=L, lens=torch.tensor(lens, dtype=torch.int32, device="cuda") if ragged else None,
                      mask=torch.from_numpy(mask).cuda())
    kk, vv = _load(kv, k, v)
    hidden = torch.from_numpy(mask == 0).cuda()[:, None, :, None]
    for t in (kv.k, kv.v, kv.k_scale, kv.v_scale):
        t.masked_fill_(hidden, 255)
    o = _attend(_ctx(H, dh, dtype), to_dev(q, dtype), kv, dtype, B, n)
    _check(f"hidden, {case}", o, kvq.attention(q, kk, vv, dh ** -0.5, lens, mask), dtype)
    if B > 1:
        assert not to_np(o)[B // 2].any()


@pytest.mark.parametrize("dtype,n", [("bf16", 1), ("bf16", 100), ("bf16", 128), ("bf16", 200), ("f32", 20)])
def test_one_workspace_serves_every_length(dtype, n):
    """The workspace of the capacity is enough for any number of rows held, whichever way that is run, and its contents do not matter."""
    B, H, dh, cap = 8, 4, 64, 6000
    ctx, kv = _ctx(H, dh, dtype), _empty_cache(B, H, cap, dh)
    kk, vv = _load(kv, _rows(10, B, cap, H, dh, dtype), _rows(11, B, cap, H, dh, dtype))
    q = _rows(12, B, n, H, dh, dtype, spread=0.2)
    size, guard = fv.fvar_kvq_attention_workspace_bytes(ctx, kv, B, n), 4096
    room = torch.empty(size + guard, dtype=torch.uint8, device="cuda")
    o = torch.empty((B, n, H, dh), dtype=to_dev(q, dtype).dtype, device="cuda")
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    for length in (0, 1, 40, 500, 1300, 3000, cap):
        for ragged in (False, True):
            held = [length] * B if not ragged else [min(cap, length + 50 * b) for b in range(B)]
            lens.copy_(torch.tensor(held, dtype=torch.int32))
            c = fv.KVQ(kv.k, kv.v, kv.k_scale, kv.v_scale, len=length, lens=lens if ragged else None)
            room.fill_(255)
            o.fill_(float("nan"))
            fv.fvar_kvq_attention(ctx, to_dev(q, dtype), c, B, n, o, room[:size])
            torch.cuda.synchronize()
            assert (room[size:] == 255).all()
            want = kvq.attention(q, kk, vv, dh ** -0.5, held)
            if length == 0 and not ragged:
                assert not to_np(o).any()
            else:
                _check(f"workspace {dtype} n {n} length {length} ragged {ragged}", o, want, dtype)


def test_one_workspace_serves_lengths_run_by_one_group_and_by_two():
    """288 blocks of 64-wide rows: in two shares each where the cache is short, 256 whole by two groups and the rest divided where it is long."""
    B, H, dh, cap, n = 8, 4, 64, 2300, 1100
    assert ways("bf16", B, n, H, H, dh, 1000, False) == (128, 4, 2) and ways("bf16", B, n, H, H, dh, cap, False) == (128, 8, 4)
    ctx, kv = _ctx(H, dh, "bf16"), _empty_cache(B, H, cap, dh)
    kk, vv = _load(kv, _rows(13, B, cap, H, dh, "bf16"), _rows(14, B, cap, H, dh, "bf16"))
    q = _rows(15, B, n, H, dh, "bf16", spread=0.2)
    size, guard = fv.fvar_kvq_attention_workspace_bytes(ctx, kv, B, n), 4096
    room = torch.empty(size + guard, dtype=torch.uint8, device="cuda")
    o = torch.empty((B, n, H, dh), dtype=torch.bfloat16, device="cuda")
    for length in (1000, 2047, 2048, cap):
        room.fill_(255)
        o.fill_(float("nan"))
        fv.fvar_kvq_attention(ctx, to_dev(q, "bf16"), fv.KVQ(kv.k, kv.v, kv.k_scale, kv.v_scale, len=length), B, n, o, room[:size])
        torch.cuda.synchronize()
        assert (room[size:] == 255).all()
        _check(f"groups, length {length}", o, kvq.attention(q, kk, vv, dh ** -0.5, [length] * B), "bf16")
