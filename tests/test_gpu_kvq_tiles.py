"""Attention over the 4-bit cache in blocks of 128 rows, in each way in which they are run (one group of wavefronts or two, whole and with the
keys divided, two wavefronts to a SIMD or three), at the places where it can go wrong: lengths, hidden rows, references that move, values,
queries and keys of every size.  The same for blocks of 16 rows where the place is theirs too.

One sample's data for two kv heads is repeated over as many samples and heads as a way takes, so that the definition in 64 bits is computed
once.  Bounds: test_gpu_kvq.py's; for scores of several hundred what a score is off by in fp32, 16 roundings of the sum of its terms' sizes, is
added to them, 2e-3 at most."""
import numpy as np
import pytest
import torch

import paper_2512_16483_amd as fv
import workloads as wl
from oracle import kvq

pytestmark = pytest.mark.gpu

from gpu_util import TOL, rel_err, tdtype, to_dev, to_np  # noqa: E402
from test_gpu_kvq import NORM, _attend, _ctx, _empty_cache, _rows  # noqa: E402
from test_kvq_tiles_host import SIXTEEN, TILES, check_way  # noqa: E402

BOTH = sorted(TILES) + sorted(SIXTEEN)


class Way:
    """A way's context and sizes, and one sample's tensors repeated over them."""

    def __init__(self, name, **kw):
        check_way(name)
        self.name = name
        self.dtype, self.dh, self.H, self.heads, self.B, self.n, self.L, *_ = {**TILES, **SIXTEEN}[name]
        self.two = min(2, self.heads)                         # kv heads of the data
        self.few = self.two * self.H // self.heads            # its query heads
        self.ctx = _ctx(self.H, self.dh, self.dtype, **kw)

    def data(self, seed, rows, heads, spread=0.5):
        return _rows(seed, 1, rows, heads, self.dh, self.dtype, spread)

    def kqv(self, seed):
        return self.data(seed, self.L, self.two), self.data(seed + 1, self.L, self.two), self.data(seed + 2, self.n, self.few, 0.2)

    def round(self, *xs):
        return [wl.round_to_bf16(x) if self.dtype == "bf16" else x.astype(np.float32) for x in xs]

    def cache(self, k, v, **kw):
        """Every sample and head with the data's rows; and the values that they stand for, [1, two, L, dh]."""
        kv, held = _empty_cache(self.B, self.heads, self.L, self.dh, len=self.L, **kw), []
        for x, codes, scales in ((k, kv.k, kv.k_scale), (v, kv.v, kv.v_scale)):
            c, s = kvq.quantise(np.swapaxes(x, 1, 2))
            for t, a in ((codes, c), (scales, s)):
                t.copy_(torch.from_numpy(a).cuda().repeat(1, self.heads // self.two, 1, 1).expand(self.B, -1, -1, -1))
            held.append(kvq.values(c, s))
        return kv, held

    def attend(self, q, kv):
        qd = to_dev(q, self.dtype).repeat(1, 1, self.H // self.few, 1).expand(self.B, -1, -1, -1).contiguous()
        return _attend(self.ctx, qd, kv, self.dtype, self.B, self.n)

    def want(self, q, held, length=None, mask=None):
        return kvq.attention(q, *held, self.dh ** -0.5, [self.L if length is None else length], mask)[0]

    def check(self, tag, got, want, off=0.0):
        """got [samples, n, H, dh], each of which should be want [n, few, dh] for all its heads; off: what is added to the bounds"""
        size = max(np.abs(want).max(), 1e-300)
        w = torch.from_numpy(np.ascontiguousarray(want / size)).cuda()[:, None]
        err = got.double().reshape(-1, self.n, self.heads // self.two, self.few, self.dh) / size - w
        rms = max(float(w.square().mean().sqrt()), 1e-300)
        norm = float(err.square().mean((1, 2, 3, 4)).sqrt().max()) / rms
        worst = float((err.abs() / w.abs().clamp_min(rms)).max())
        print(f"[kvq] {self.name} {tag}: norm {norm:.3g} max {worst:.3g}", flush=True)
        assert norm <= NORM[self.dtype] + off and worst <= TOL[self.dtype] + off, (tag, norm, worst)


def _off(way, q, kk, vv, want):
    """Bound on how far fp32 scores take a result: 2 * 16 * 2^-24 * the largest sum of |q| |k|, times the spread of the values, relative to
    the result."""
    s = way.dh ** -0.5 * np.einsum("nhd,htd->hnt", np.abs(q[0]).astype(np.float64), np.repeat(np.abs(kk[0]), way.few // way.two, 0)).max()
    return 2 * 16 * 2.0 ** -24 * s * np.abs(vv).max() / np.sqrt(np.mean(want ** 2))


# ------------------------------------------------------------------------------------ lengths and masks
@pytest.mark.parametrize("name", sorted(TILES))
def test_every_kind_of_length(name):
    way = Way(name)
    lengths = [0, 1, 2, 15, 31, 32, 33, 63, 64, 65, 127, 128, 129, 191, 192, 193, 255, 256, 257, way.L - 1, way.L]
    k, v, q = way.kqv(10)
    lens = torch.zeros(way.B, dtype=torch.int32, device="cuda")
    for at in range(0, len(lengths), way.B):
        some = (lengths[at:at + way.B] * way.B)[:way.B]
        kv, held = way.cache(k, v, lens=lens)
        lens.copy_(torch.tensor(some, dtype=torch.int32))
        for b, length in enumerate(some):                     # what lies behind a sample's rows is not a number
            kv.k_scale[b, :, length:], kv.v_scale[b, :, length:] = 255, 255
        o = way.attend(q, kv)
        for length in sorted(set(some)):
            mine = o[[i for i, x in enumerate(some) if x == length]]
            if length == 0:
                assert not mine.any()
            else:
                way.check(f"length {length}", mine, way.want(q, held, length))


@pytest.mark.parametrize("name", sorted(TILES))
def test_every_kind_of_mask(name):
    way = Way(name)
    t, g = np.arange(way.L), np.random.default_rng(30)
    masks = [np.ones(way.L), g.random(way.L) < 0.7, g.random(way.L) < 0.02, np.zeros(way.L), t == 0, t == way.L - 1, t >= 320, t < 64,
             (t // 64) % 2, (t // 64) % 2 == 0, (t // 32) % 2, t == 333, t // 64 == way.L // 64, (t < 100) | (t >= 400)]
    one = {4: 0, 5: way.L - 1, 11: 333}
    k, v, q = way.kqv(31)
    for at in range(0, len(masks), way.B):
        some = [(at + i % min(way.B, len(masks) - at)) for i in range(way.B)]
        mask = np.array([masks[i] for i in some]).astype(np.uint8) * 255
        kv, held = way.cache(k, v, mask=torch.from_numpy(mask).cuda())
        hidden = torch.from_numpy(mask == 0).cuda()[:, None, :, None]
        for x in (kv.k, kv.v, kv.k_scale, kv.v_scale):
            x.masked_fill_(hidden, 255)
        o = way.attend(q, kv)
        for i in sorted(set(some)):
            mine, want = o[[b for b, x in enumerate(some) if x == i]], way.want(q, held, mask=masks[i][None])
            if i == 3:
                assert not mine.any()
            elif i in one:                                    # its values, which are exact
                w = torch.from_numpy(want).to(o.dtype).cuda()
                assert (w.double().cpu().numpy() == want).all() and (mine.reshape(-1, way.n, way.H // way.few, way.few, way.dh) == w[:, None]).all()
            else:
                way.check(f"mask {i}", mine, want)


# ------------------------------------------------------------------------------------ what is not a number
@pytest.mark.parametrize("name", sorted(TILES))
def test_what_is_not_a_number_is_passed_on(name):
    """A NaN in a visible value, key or query makes exactly the outputs NaN that it takes part in; so does an infinite query."""
    way = Way(name)
    k, v, q = way.kqv(40)
    kv, held = way.cache(k, v)
    G, last = way.H // way.heads, way.L - 1
    kv.v_scale[1, 0, 70, 1] = 255
    kv.k_scale[2, way.heads - 1, last, 0] = 255
    qd = to_dev(q, way.dtype).repeat(1, 1, way.H // way.few, 1).repeat(way.B, 1, 1, 1)
    qd[3, way.n - 1, way.H - 1, 5], qd[0, 0, 0, way.dh - 1], qd[0, 7, 0, 40] = float("nan"), float("inf"), float("-inf")
    o = to_np(_attend(way.ctx, qd, kv, way.dtype, way.B, way.n))
    bad = np.zeros(o.shape, bool)
    bad[1, :, :G, 32:64] = bad[2, :, way.H - G:] = bad[3, way.n - 1, way.H - 1] = bad[0, 0, 0] = bad[0, 7, 0] = True
    assert np.array_equal(np.isnan(o), bad)
    want = np.tile(way.want(q, held), (1, way.H // way.few, 1))
    for b in range(min(4, way.B)):
        w = np.where(bad[b], 0, want)
        got = np.where(bad[b], 0, o[b])
        norm, worst = np.linalg.norm(got - w) / np.linalg.norm(w), rel_err(got, w)
        assert norm <= NORM["bf16"] and worst <= TOL["bf16"], (b, norm, worst)


# ------------------------------------------------------------------------------------ sizes
@pytest.mark.parametrize("name", BOTH)
@pytest.mark.parametrize("case", ["sharp", "rising", "falling", "steps", "steps down", "queries of every size", "some large queries"])
def test_references_that_move(name, case):
    """Scores of several hundred, which rise or fall along the rows, a little at every row or much at some: the running reference has to be
    found anew again and again, in rows of a block at different places."""
    way = Way(name)
    k, v, q = way.kqv(50)
    t = np.arange(way.L)
    if case == "sharp":
        q = q * 8
    elif case == "queries of every size":                     # rows of a block whose references lie far apart
        q = q * 2.0 ** np.random.default_rng(55).integers(-12, 5, (1, way.n, way.few, 1))
    elif case == "some large queries":                        # those of one wavefront, with keys that grow
        q = q * np.where(np.arange(way.n) // 32 % 4 == 1, 30.0, 1.0)[None, :, None, None]
        k = k * 2.0 ** (t // 150 % 3 - 1.0)[None, :, None, None]
    else:
        up = {"rising": 2.0 ** np.linspace(-10, 4, way.L), "steps": 2.0 ** (t // 97 % 7 - 3.0)}.get(case.split(" down")[0], None)
        if case == "falling":
            up = 2.0 ** np.linspace(4, -10, way.L)
        if case == "steps down":
            up = up[::-1]
        q, k = np.abs(q), np.abs(k) * up[None, :, None, None]
    k, q = way.round(k, q)
    kv, held = way.cache(k, v)
    o, want = way.attend(q, kv), way.want(q, held)
    way.check(case, o, want, min(_off(way, q, *held, want), 2e-3))


@pytest.mark.parametrize("name", BOTH)
@pytest.mark.parametrize("case", ["tiny values", "huge values", "largest values", "mixed values", "rising values", "tiny queries", "huge queries",
                                  "huge keys"])
def test_values_queries_and_keys_of_every_size(name, case):
    way = Way(name)
    k, v, q = way.kqv(60)
    g = np.random.default_rng(63)
    if case == "tiny values":
        v = v * 2.0 ** -110
    elif case == "huge values":
        v = v * 2.0 ** 115
    elif case == "largest values":                            # a mean of some that are near the largest number is not past it
        v = np.sign(v) * 3e38 * (1 - 0.2 * g.random(v.shape))
    elif case == "mixed values":                              # sizes from 2^-30 to 1, in no order
        v = v * 2.0 ** -g.integers(0, 31, (1, way.L, way.two, 1))
    elif case == "rising values":                             # each tile's larger than the one's before
        v = v * 2.0 ** np.linspace(-24, 8, way.L)[None, :, None, None]
    elif case == "tiny queries":
        q = q * 2.0 ** -100
    elif case == "huge queries":
        q, k = q * 2.0 ** 80, k * 2.0 ** -80
    elif case == "huge keys":
        q, k = q * 2.0 ** -90, k * 2.0 ** 90
    k, v, q = way.round(k.astype(np.float32), v.astype(np.float32), q.astype(np.float32))
    kv, held = way.cache(k, v)
    o, want = way.attend(q, kv), way.want(q, held)
    way.check(case, o, want)


@pytest.mark.parametrize("name", sorted(TILES))
def test_equal_scores_are_the_mean(name):
    way = Way(name)
    k, v, q = way.kqv(70)
    kv, held = way.cache(k, v)
    o, want = to_np(way.attend(np.zeros_like(q), kv)[:2]).reshape(2, way.n, -1, way.two, way.few // way.two, way.dh), held[1].mean(2)[0][:, None]
    lim = 2.0 ** -8 * np.abs(want) + way.L * 2.0 ** -24 * np.abs(held[1]).mean(2)[0][:, None]
    assert (np.abs(o - want) <= lim).all()


@pytest.mark.parametrize("name", BOTH)
@pytest.mark.parametrize("scale", [1e-30, 1.3e-38, 2e-38])
def test_a_scale_that_makes_all_scores_equal(name, scale):
    way = Way(name, attn_scale=scale)
    k, v, q = way.kqv(74)
    kv, held = way.cache(k, v)
    want = np.repeat(held[1][0].mean(1), way.few // way.two, 0)[None]
    way.check(f"scale {scale}", way.attend(q, kv), np.tile(want, (way.n, 1, 1)))


@pytest.mark.parametrize("name", BOTH)
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_of_every_size(name, sign):
    """Two kinds of keys, one with twice the other's score, about 2^size: all weight lies on the larger score's, equally, and the result is the mean
    of their values, whichever tiles, shares and groups they stand in."""
    way = Way(name)
    g, t = np.random.default_rng(71), np.arange(way.L)
    unit = np.where(g.random(way.dh) < 0.5, -1.0, 1.0)        # scores are sums of equal terms, without rounding
    kind = np.where(t * 7 // 3 % 5 < 3, 2.0, 1.0)
    if sign < 0:                                              # the larger score in few places, the last tile's and the first's among others
        kind = np.where(np.isin(t, [3, 4, way.L // 2, way.L - 1]), 1.0, 2.0)
    _, v, _ = way.kqv(72)
    for size in (20, 24, 26, 27, 28, 30, 40, 60, 100, 112):
        half = size // 2
        k = (kind[:, None] * unit)[None, :, None] * 2.0 ** half * np.ones((1, 1, way.two, 1))
        q = sign * unit * 2.0 ** (size - half) / way.dh ** 0.5 * np.ones((1, way.n, way.few, 1))
        k, q = way.round(k.astype(np.float32), q.astype(np.float32))
        kv, held = way.cache(k, v)
        want = np.repeat(held[1][0][:, kind == (2 if sign > 0 else 1)].mean(1), way.few // way.two, 0)[None]
        way.check(f"scores {sign * 2.0 ** size:.1g}", way.attend(q, kv), np.tile(want, (way.n, 1, 1)))


# ------------------------------------------------------------------------------------ queries with elements of very different sizes
@pytest.mark.parametrize("name", BOTH)
@pytest.mark.parametrize("case", ["x 30", "x 200", "x 1000", "x 1e5", "half of them", "one to a block", "a ladder"])
def test_queries_with_elements_far_larger_than_the_others(name, case):
    """Scores of about 15 that come from a query's small elements, where the keys of its largest are 0 or small: each element counts with all
    bits that it was given with."""
    way = Way(name)
    k, v, q = way.kqv(80)
    g = np.random.default_rng(83)
    q = q * 4
    lift = np.ones(way.dh)
    if case.startswith("x"):
        lift[g.integers(0, way.dh)] = float(case[2:])
    elif case == "half of them":
        lift[g.permutation(way.dh)[:way.dh // 2]] = 2000.0
    elif case == "one to a block":
        lift[5::32] = 700.0
    else:
        lift = 2.0 ** (np.arange(way.dh) % 32 / 2)            # 1 to 2^15 in every block
    q, k = way.round((q * lift).astype(np.float32), (k / lift).astype(np.float32))
    kv, held = way.cache(k, v)
    o, want = way.attend(q, kv), way.want(q, held)
    way.check(case, o, want, min(_off(way, q, *held, want), 2e-3))


# ------------------------------------------------------------------------------------ a graph
@pytest.mark.parametrize("name", ["two groups, 128", "two groups divided, 64", "one group, 64, 3 waves"])
def test_a_captured_graph(name):
    """Append and attention as nodes of a graph, replayed with new rows and lengths between other work."""
    way = Way(name)
    new = 16
    cap = way.L
    lens, total = (torch.zeros(way.B, dtype=torch.int32, device="cuda") for _ in range(2))
    k, v, q = way.kqv(90)
    kv, _ = way.cache(k, v, lens=lens)
    after = fv.KVQ(kv.k, kv.v, kv.k_scale, kv.v_scale, lens=total)
    kd, vd = (torch.zeros((way.B, new, way.heads, way.dh), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    qd = torch.zeros((way.B, way.n, way.H, way.dh), dtype=torch.bfloat16, device="cuda")
    o = torch.empty_like(qd)
    ws = torch.empty(fv.fvar_kvq_attention_workspace_bytes(way.ctx, after, way.B, way.n), dtype=torch.uint8, device="cuda")

    def step():
        fv.fvar_kvq_append(way.ctx, kv, kd, vd, way.B, new)
        fv.fvar_kvq_attention(way.ctx, qd, after, way.B, way.n, o, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for r in range(3):
        held = [max(0, cap - new - 50 * r - 10 * b) for b in range(way.B)]
        lens.copy_(torch.tensor(held, dtype=torch.int32))
        total.copy_(lens + new)
        for i, t in enumerate((kd, vd, qd)):
            x = to_dev(way.data(92 + 3 * r + i, t.shape[1], way.two if i < 2 else way.few), "bf16")
            t.copy_(x.repeat(1, 1, t.shape[2] // x.shape[2], 1).expand(way.B, -1, -1, -1))
        o.fill_(float("nan"))
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        got = o.clone()
        vals = [kvq.values(c[:1, :way.two].cpu().numpy(), s[:1, :way.two].cpu().numpy()) for c, s in ((kv.k, kv.k_scale), (kv.v, kv.v_scale))]
        way.check(f"graph, replay {r}", got[:1], way.want(to_np(qd[:1, :, :way.few]), vals, held[0] + new))
        o.fill_(float("nan"))
        step()
        torch.cuda.synchronize()
        assert torch.equal(o, got)
