"""The operators of a key/value cache held in 8 bits, by which their speed and outputs are judged: rotary positions on their way into
it, the cache and the attention that reads it, and the eviction of rows by the attention weight that they have gathered.

A program that generates images scale by scale keeps the keys and values of every scale, and one that generates text those of every
token.  Per block and step, queries and keys are turned by their positions ("rope"), keys and values are written to the cache in 8 bits
("write", which also reads them back), the queries attend over it ("attend", which can also return the weight that every row has got), and
when the cache has grown too long the rows that got the least are dropped ("evict", which also reads back what is left).

Rotary positions: the first `dim` elements of a head are `axes` parts of P = dim / axes; part a is turned by component a of the row's
position, pair i of P / 2 by the angle position * f_i, f_i = base^(-2 i / P).  A pair is the elements (i, i + P / 2) of the part, or
(2 i, 2 i + 1) where interleaved.  Longer contexts than the model was trained for: "linear" f_i / s; "ntk" base * s^(P / (P - 2)) in place of base;
"yarn" f_i (g_i + (1 - g_i) / s), where g_i = clamp((r_i - low) / (high - low), 0, 1) of the turns r_i = original * f_i / (2 pi), cosine and sine
times a magnitude.

Cache: elements in E4M3 (sign, 4 bits of exponent with bias 7, 3 of mantissa, up to 448; 127 is NaN), which share a power of two 2^e, stored as the byte
e + 127, over a block of 32 consecutive rows of one head.  e is the smallest integer within [-117, 119] with max |x| <= 464 * 2^e over the
finite elements; an element is the nearest value, ties to the even code, at most 448; what is not finite is NaN.  Rows written into a block that holds some
raise its e where they have to, and the ones that it holds are rounded to the new one.
    codes  uint8 [batch, kv_heads, capacity, head_dim]
    scales uint8 [batch, kv_heads, ceil(capacity / 32)]

Eviction, per sample and kv head: of the rows that a sample holds and that are not hidden, `keep` stay: the last `recent` of all that it holds, and of the
others those with the largest weights, equal ones from the lowest row on.  They move to the front in their order; a block's e is the smallest
for what it then holds.

Sizes are those of the workloads in `workloads/` (see perf/cases.py), with fewer kv heads than query heads as the generic
case; `draw` spreads over the same ranges, odd sizes included.
"""
from __future__ import annotations

import math

import torch

own = False

# heads, head_dim of the model shapes in `workloads/`
GEOMETRY = {"d1024": (16, 64), "d1920": (30, 64), "d2048": (16, 128), "d4096": (32, 128)}
BLOCK = 32


def _rope(model, kv_heads, batch, rows, dim, layout, axes=1, scaling="none", far=0, dtype="bf16"):
    return dict(kind="rope", model=model, kv_heads=kv_heads, batch=batch, rows=rows, dim=dim, layout=layout, axes=axes, scaling=scaling,
                far=far, dtype=dtype)


def _write(model, kv_heads, batch, rows, prefix, dtype="bf16", ragged=False):
    return dict(kind="write", model=model, kv_heads=kv_heads, batch=batch, rows=rows, prefix=prefix, dtype=dtype, ragged=ragged)


def _attend(model, kv_heads, batch, queries, keys, dtype="bf16", ragged=False, masked=False, weights=False):
    return dict(kind="attend", model=model, kv_heads=kv_heads, batch=batch, queries=queries, keys=keys, dtype=dtype, ragged=ragged,
                masked=masked, weights=weights)


def _evict(model, kv_heads, batch, keys, keep, recent, dtype="bf16", ragged=False, masked=False):
    return dict(kind="evict", model=model, kv_heads=kv_heads, batch=batch, keys=keys, keep=keep, recent=recent, dtype=dtype, ragged=ragged,
                masked=masked)


def listed():
    cases = {
        # one token each of a serving step far behind the trained context, grouped heads: latency
        "rope_tokens_b32": _rope("d4096", 8, 32, 1, 128, "interleaved", scaling="yarn", far=1000000),
        # the kept rows of the 80x80 scale, batch 4: positions on the grid
        "rope_grid_large": _rope("d4096", 32, 4, 1600, 128, "half", axes=2),
        # 32-bit storage, half of every head turned, an odd number of rows
        "rope_part_f32": _rope("d1024", 16, 2, 553, 32, "half", scaling="ntk", far=40000, dtype="f32"),
        # one token each of 32 sequences of different lengths, grouped heads: a serving step
        "write_tokens_b32": _write("d4096", 8, 32, 1, 16920, ragged=True),
        # every token of the 80x80 scale, batch 4, behind all earlier ones
        "write_large": _write("d4096", 32, 4, 6400, 10521),
        # one query of a single image over the whole cache: latency and the split of a long axis
        "attend_token_b1": _attend("d2048", 16, 1, 1, 10521),
        # a serving step: one query each of 32 sequences of different lengths (one of them empty), some rows hidden, with the rows' weights
        "attend_tokens_b32": _attend("d4096", 8, 32, 1, 16921, ragged=True, masked=True, weights=True),
        # a serving batch: kept rows of the 40x40 scale, 16 images with guidance doubling, with the rows' weights for the next eviction
        "attend_b32": _attend("d2048", 16, 32, 480, 3001, weights=True),
        # the largest shape: kept rows of the 80x80 scale over all earlier ones
        "attend_large": _attend("d4096", 32, 4, 1600, 12121),
        # 32-bit storage, head_dim 64, a mask over the rows, with their weights
        "attend_f32": _attend("d1024", 16, 2, 128, 552, dtype="f32", masked=True, weights=True),
        # the cache of a single image down to 0.4 of its rows: latency
        "evict_b1": _evict("d2048", 16, 1, 10521, 4209, 256),
        # 4 sequences of different lengths, some rows hidden, down to half of the longest
        "evict_large": _evict("d4096", 32, 4, 16921, 8461, 1024, ragged=True, masked=True),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "write", "attend", "attend", "attend", "evict"])
    model = rng.choice(list(GEOMETRY))
    heads, dh = GEOMETRY[model]
    kv_heads = heads // rng.choice([g for g in (1, 1, 1, 2, 3, 4, 8) if heads % g == 0])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    batch = _log_int(rng, 1, 32)
    if kind == "rope":
        axes = rng.choice([1, 1, 2])
        rows, dim = _log_int(rng, 1, 6400), 16 * axes * rng.randint(1, dh // 16 // axes)
        while batch * rows * (heads + kv_heads) * dh > 5e7:
            batch, rows = max(1, batch // 2), rows if batch > 1 else rows // 2
        scaling = rng.choice(["none", "linear", "ntk", "yarn"] if dim > 16 * axes else ["none", "linear", "yarn"])
        return _rope(model, kv_heads, batch, rows, dim, rng.choice(["half", "interleaved"]), axes, scaling,
                     _log_int(rng, 1, 1000000) if axes == 1 else 0, dtype)
    if kind == "write":
        rows = _log_int(rng, 1, 6400)
        while batch * rows * kv_heads * dh > 5e7:
            batch, rows = max(1, batch // 2), rows if batch > 1 else rows // 2
        return _write(model, kv_heads, batch, rows, _log_int(rng, 1, 10521), dtype, rng.random() < 0.5)
    if kind == "evict":
        keys = _log_int(rng, 2, 16921)
        while batch * kv_heads * keys * dh > 2.5e8:
            batch, keys = max(1, batch // 2), keys if batch > 1 else keys // 2
        keep = max(1, int(keys * rng.uniform(0.05, 1.0)))
        return _evict(model, kv_heads, batch, keys, keep, int(keep * rng.uniform(0.0, 1.0)), dtype, rng.random() < 0.4, rng.random() < 0.4)
    queries, keys = _log_int(rng, 1, 1600), _log_int(rng, 1, 16921)
    if dtype == "f32":
        queries, keys = min(queries, 256), max(1, keys // 8)
    weights = rng.random() < 0.5
    while batch * heads * queries * keys > (8e8 if weights else 1.2e9) or batch * kv_heads * keys * dh > 4e8:
        if batch > 1:
            batch //= 2
        else:
            queries, keys = max(1, queries * 3 // 4), max(1, keys * 3 // 4)
    return _attend(model, kv_heads, batch, queries, keys, dtype, rng.random() < 0.4, rng.random() < 0.3, weights)


# ------------------------------------------------------------------------------------ inputs
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _lengths(case, longest):
    """Rows of each sample's cache: from the longest downwards, and none at all for the last of four or more."""
    B = case["batch"]
    if not case.get("ragged"):
        return [longest] * B
    return [longest - b * longest // B if b < 3 or b < B - 1 else 0 for b in range(B)]


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _rows(g, batch, rows, heads, dh, dt):
    """New rows as a projection leaves them: channels of different sizes."""
    return (_randn(g, batch, rows, heads, dh) * torch.exp(0.3 * _randn(g, heads, dh))).to(dt)


def _cache(g, batch, heads, capacity, dh, dt):
    """Codes and scales of `capacity` rows per sample."""
    blocks = -(-capacity // BLOCK)
    codes = torch.empty((batch, heads, capacity, dh), dtype=torch.uint8, device="cuda")
    scales = torch.empty((batch, heads, blocks), dtype=torch.uint8, device="cuda")
    for b in range(batch):
        x = _rows(g, 1, blocks * BLOCK, heads, dh, dt)[0].transpose(0, 1).float().reshape(heads, blocks, BLOCK, dh)
        x.reshape(heads, -1, dh)[:, capacity:] = 0
        e = _exponent(x)
        codes[b] = _encode(x, e).reshape(heads, -1, dh)[:, :capacity]
        scales[b] = (e + 127).to(torch.uint8)
    return codes, scales


def _rope_settings(case):
    """What a model's configuration says of its rotary positions."""
    s = dict(dim=case["dim"], interleaved=case["layout"] == "interleaved", axes=case["axes"], base=10000.0, scaling=case["scaling"])
    if case["scaling"] != "none":
        s["factor"] = 8.0
    if case["scaling"] == "yarn":
        s.update(original=4096.0, low=1.0, high=32.0, magnitude=0.1 * math.log(8.0) + 1.0)
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    heads, dh = GEOMETRY[case["model"]]
    hk, B, dt = case["kv_heads"], case["batch"], _dtype(case)
    s = dict(case=case)

    def buf(*shape, dtype=dt):
        return torch.empty(shape, dtype=dtype, device="cuda")

    if case["kind"] == "rope":
        n = case["rows"]
        fused = _randn(g, B, n, heads + 2 * hk, dh).to(dt)          # the output of one projection to queries, keys and values
        s.update(fused=fused, q=fused[:, :, :heads], k=fused[:, :, heads:heads + hk], q_out=buf(B, n, heads, dh), k_out=buf(B, n, hk, dh))
        if case["axes"] == 1:                                      # sequences that stand at different positions
            start = torch.randint(case["far"] // 2, case["far"] + 1, (B, 1), generator=g, device="cuda")
            s["pos"] = (start + torch.arange(n, device="cuda")).to(torch.int32)
        else:                                                      # the rows kept of a token map, in their order
            side = math.isqrt(4 * n - 1) + 1
            kept = torch.rand((B, side * side), generator=g, device="cuda").argsort(-1)[:, :n].sort(-1).values
            s["pos"] = torch.stack([kept // side, kept % side], -1).to(torch.int32)
        return s
    if case["kind"] == "write":
        held = -(-case["prefix"] // BLOCK) * BLOCK
        capacity = held + -(-case["rows"] // BLOCK) * BLOCK + BLOCK
        for n in ("k", "v"):
            s[n] = _rows(g, B, case["rows"], hk, dh, dt).contiguous()
            codes, scales = _cache(g, B, hk, held, dh, dt)
            s[n + "_codes"] = torch.cat([codes, torch.zeros((B, hk, capacity - held, dh), dtype=torch.uint8, device="cuda")], 2)
            s[n + "_scale"] = torch.cat([scales, torch.zeros((B, hk, (capacity - held) // BLOCK), dtype=torch.uint8, device="cuda")], 2)
            s[n + "_back"] = buf(B, case["rows"] + BLOCK - 1, hk, dh)
        s["first"] = torch.tensor(_lengths(case, case["prefix"]), dtype=torch.int32, device="cuda")
        s["last"] = s["first"] + case["rows"]
        return s
    capacity = case["keys"]
    for n in ("k", "v"):
        s[n + "_codes"], s[n + "_scale"] = _cache(g, B, hk, capacity, dh, dt)
    s["lens"] = torch.tensor(_lengths(case, capacity), dtype=torch.int32, device="cuda") if case["ragged"] else None
    s["mask"] = (torch.rand((B, capacity), generator=g, device="cuda") < 0.7).to(torch.uint8) if case["masked"] else None
    if case["kind"] == "attend":
        s["q"] = _randn(g, B, case["queries"], heads, dh).to(dt)
        s["o"] = buf(B, case["queries"], heads, dh)
        s["weights"] = torch.zeros((B, hk, capacity), device="cuda") if case["weights"] else None
        return s
    # Weights as attention leaves them: a few rows have most; rows that came last have had little time; some have got nothing at all.
    s["weights"] = torch.exp(2 * _randn(g, B, hk, capacity)) * (torch.rand((B, hk, capacity), generator=g, device="cuda") < 0.9)
    keep = case["keep"]
    s.update(to_weights=buf(B, hk, keep, dtype=torch.float32), to_lens=buf(B, dtype=torch.int32), idx=buf(B, hk, keep, dtype=torch.int32))
    for n in ("k", "v"):
        s["to_" + n] = buf(B, hk, keep, dh, dtype=torch.uint8)
        s["to_" + n + "_scale"] = buf(B, hk, -(-keep // BLOCK), dtype=torch.uint8)
        s[n + "_back"] = buf(B, keep, hk, dh)
    return s


def work(case):
    heads, dh = GEOMETRY[case["model"]]
    hk, B = case["kv_heads"], case["batch"]
    es = 2 if case["dtype"] == "bf16" else 4
    held = dh + 1 / BLOCK                                          # bytes of one row of one head
    if case["kind"] == "rope":
        rows = B * case["rows"]
        return {"bytes": 2 * rows * (heads + hk) * dh * es + 4 * rows * case["axes"], "flops": 3.0 * rows * (heads + hk) * case["dim"]}
    if case["kind"] == "write":
        rows = 2 * B * case["rows"] * hk                            # K and V
        return {"bytes": 2 * rows * (dh * es + held), "flops": 0}
    keys = sum(_lengths(case, case["keys"]))
    seen = 0.7 * keys if case["masked"] else keys
    if case["kind"] == "evict":
        kept = sum(min(case["keep"], 0.7 * n if case["masked"] else n) for n in _lengths(case, case["keys"])) * hk
        moved = 2 * kept * (2 * held + held + dh * es)              # read and written by the eviction, read and written again by the reading
        return {"bytes": moved + 4 * keys * hk + 8 * kept + (keys if case["masked"] else 0), "flops": 0}
    qo = 2 * B * case["queries"] * heads * dh * es
    both = 6.0 if case["weights"] else 4.0                         # the weights need every row's total before, so the scores twice
    return {"bytes": qo + 2 * seen * hk * held + (keys if case["masked"] else 0) + (4 * keys * hk if case["weights"] else 0),
            "flops": both * seen * case["queries"] * heads * dh}


# ------------------------------------------------------------------------------------ plain form
def _power(e):
    """2^e for int32 tensors of exponents of normal numbers."""
    return ((e + 127) << 23).view(torch.float32)


def _exponent(x):
    """The e of blocks x [..., rows, dh] of fp32 numbers: the smallest with max |x| <= 464 * 2^e."""
    top = torch.where(torch.isfinite(x), x.abs(), 0.0).amax((-2, -1))
    m, e = torch.frexp(top)                                        # top = m 2^e, m in [.5, 1); 464 = .90625 * 2^9
    e = (e - 9 + (m > 0.90625).to(torch.int32)).clamp(-117, 119)
    return torch.where(top == 0, -117, e)


def _encode(x, e):
    """Codes of x [..., rows, dh] with the blocks' e [...]."""
    half = torch.div(-e, 2, rounding_mode="floor")                  # (2^-e in two factors, each a normal number)
    y = x * _power(half)[..., None, None] * _power(-e - half)[..., None, None]
    y = torch.where(torch.isfinite(x), y.clamp(-448.0, 448.0), float("nan"))
    codes = y.to(torch.float8_e4m3fn).view(torch.uint8)
    return torch.where(torch.isfinite(x), codes, 127)


def _values(codes, scales):
    """The values that codes [..., capacity, dh] and scales [..., blocks] stand for, in 32 bits."""
    size = _power(scales.to(torch.int32) - 127).repeat_interleave(BLOCK, -1)[..., :codes.shape[-2]]
    return codes.view(torch.float8_e4m3fn).float() * size.unsqueeze(-1)


def _plain_rope(s):
    case = s["case"]
    r, dt = _rope_settings(case), _dtype(case)
    part = r["dim"] // r["axes"]
    i = torch.arange(part // 2, device="cuda", dtype=torch.float64)
    base, factor = r["base"], r.get("factor", 1.0)
    if r["scaling"] == "ntk":
        base = base * factor ** (part / (part - 2))
    f = base ** (-2.0 * i / part)
    if r["scaling"] == "linear":
        f = f / factor
    if r["scaling"] == "yarn":
        keep = ((r["original"] * f / (2 * math.pi) - r["low"]) / (r["high"] - r["low"])).clamp(0.0, 1.0)
        f = f * (keep + (1 - keep) / factor)
    pos = s["pos"] if r["axes"] == 2 else s["pos"].unsqueeze(-1)
    angle = pos.double().unsqueeze(-1) * f                          # [B, n, axes, part / 2]: in 64 bits, far positions need them
    size = r.get("magnitude", 1.0)
    cos, sin = (size * angle.cos()).float().unsqueeze(2), (size * angle.sin()).float().unsqueeze(2)
    out = {}
    for name in ("q", "k"):
        x = s[name].float()
        y = x[..., :r["dim"]].unflatten(-1, (r["axes"], part))
        if r["interleaved"]:
            a, b = y[..., 0::2], y[..., 1::2]
            y = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
        else:
            a, b = y[..., :part // 2], y[..., part // 2:]
            y = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
        out[name] = torch.cat([y.flatten(-2), x[..., r["dim"]:]], -1).to(dt)
    return out


def _plain_write(s):
    case = s["case"]
    B, rows, hk, dh = s["k"].shape
    blocks = (rows + 2 * BLOCK - 2) // BLOCK                       # as many as the rows can touch
    first = s["first"].long()
    block = first[:, None] // BLOCK + torch.arange(blocks, device="cuda")             # [B, blocks]
    at = (first // BLOCK * BLOCK)[:, None] + torch.arange(blocks * BLOCK, device="cuda")
    j = at - first[:, None]
    new, old = ((j >= 0) & (j < rows))[:, None, :, None], (j < 0)[:, None, :, None]
    back = first[:, None] + torch.arange(1 - BLOCK, rows, device="cuda")
    out = {}
    for n in ("k", "v"):
        codes, scales = s[n + "_codes"], s[n + "_scale"]
        here = at[:, None, :, None].expand(B, hk, blocks * BLOCK, dh)
        which = block[:, None].expand(B, hk, blocks)
        c, e = codes.gather(2, here), scales.gather(2, which).to(torch.int32) - 127
        incoming = s[n].transpose(1, 2).float().gather(2, j.clamp(0, rows - 1)[:, None, :, None].expand_as(here))
        incoming = torch.where(new, incoming, 0.0).unflatten(2, (blocks, BLOCK))
        holds = old.unflatten(2, (blocks, BLOCK)).any(3).any(-1)
        wanted = torch.where(holds, torch.maximum(e, _exponent(incoming)), _exponent(incoming))
        kept = (c.view(torch.float8_e4m3fn).float().unflatten(2, (blocks, BLOCK)) * _power(torch.where(holds, e, 0))[..., None, None])
        kept = torch.where(old.unflatten(2, (blocks, BLOCK)), kept, 0.0)
        mixed = torch.where(old, _encode(kept, wanted).flatten(2, 3), torch.where(new, _encode(incoming, wanted).flatten(2, 3), c))
        codes.scatter_(2, here, mixed)
        touched = new.unflatten(2, (blocks, BLOCK)).any(3).any(-1)
        scales.scatter_(2, which, torch.where(touched, wanted + 127, e + 127).to(torch.uint8))
        there = (back >= 0)[:, None, :, None]
        values = codes.gather(2, back.clamp_min(0)[:, None, :, None].expand(B, hk, -1, dh)).view(torch.float8_e4m3fn).float()
        size = _power(scales.gather(2, (back.clamp_min(0) // BLOCK)[:, None].expand(B, hk, -1)).to(torch.int32) - 127)
        out[n] = torch.where(there, values * size.unsqueeze(-1), 0.0).transpose(1, 2).to(_dtype(case)).contiguous()
    return out


def _seen(s):
    case = s["case"]
    B, L = case["batch"], case["keys"]
    seen = torch.ones((B, L), dtype=torch.bool, device="cuda")
    if s["lens"] is not None:
        seen = seen & (torch.arange(L, device="cuda") < s["lens"][:, None])
    return seen if s["mask"] is None else seen & (s["mask"] != 0)


def _plain_attend(s):
    case = s["case"]
    dt = _dtype(case)
    heads, dh = GEOMETRY[case["model"]]
    B, n, hk = case["batch"], case["queries"], case["kv_heads"]
    k, v = _values(s["k_codes"], s["k_scale"]), _values(s["v_codes"], s["v_scale"])
    q = s["q"].float().reshape(B, n, hk, heads // hk, dh).permute(0, 2, 3, 1, 4).reshape(B, hk, -1, dh)
    x = torch.matmul(q, k.transpose(-1, -2).contiguous()) * dh ** -0.5
    if s["lens"] is not None or s["mask"] is not None:
        seen = _seen(s)
        x = torch.where(seen[:, None, None], x, -math.inf)
        v = torch.where(seen[:, None, :, None], v, 0.0)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    o = torch.matmul(p, v)
    o = o.reshape(B, hk, heads // hk, n, dh).permute(0, 3, 1, 2, 4).reshape(B, n, heads, dh).to(dt)
    return {"o": o, "weights": p.sum(2, dtype=torch.float64).float()} if case["weights"] else {"o": o}


def _plain_evict(s):
    case = s["case"]
    B, L, keep, hk = case["batch"], case["keys"], case["keep"], case["kv_heads"]
    _, dh = GEOMETRY[case["model"]]
    at = torch.arange(L, device="cuda")
    lens = s["lens"] if s["lens"] is not None else torch.full((B,), L, device="cuda")
    seen = _seen(s)
    rank = torch.where((at >= (lens - case["recent"])[:, None])[:, None], math.inf, s["weights"])
    rank = torch.where(seen[:, None], rank, -math.inf)
    order = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :keep]
    count = seen.sum(-1).clamp_max(keep)
    there = (torch.arange(keep, device="cuda") < count[:, None])[:, None].expand(B, hk, keep)
    idx = torch.where(there, order, L).sort(-1).values
    src = idx.clamp_max(L - 1)
    blocks = -(-keep // BLOCK)
    out = {"idx": torch.where(there, idx, -1).to(torch.int32), "lens": count.to(torch.int32),
           "weights": torch.where(there, s["weights"].gather(-1, src), 0.0)}
    for n in ("k", "v"):
        x = _values(s[n + "_codes"], s[n + "_scale"]).gather(2, src.unsqueeze(-1).expand(-1, -1, -1, dh))
        x = torch.where(there.unsqueeze(-1), x, 0.0)
        x = torch.cat([x, x.new_zeros((B, hk, blocks * BLOCK - keep, dh))], 2).unflatten(2, (blocks, BLOCK))
        e = _exponent(x)
        back = _encode(x, e).view(torch.float8_e4m3fn).float() * _power(e)[..., None, None]
        out[n] = back.flatten(2, 3)[:, :, :keep].transpose(1, 2).to(_dtype(case)).contiguous()
    return out


def _plain(s):
    return {"rope": _plain_rope, "write": _plain_write, "attend": _plain_attend, "evict": _plain_evict}[s["case"]["kind"]](s)


# ------------------------------------------------------------------------------------ the framework's own form
def _handle(s):
    """What a program keeps from call to call: the model's context, the caches' handles, a call's workspace."""
    if "handle" not in s:
        import paper_2512_16483_amd as fv
        case = s["case"]
        heads, dh = GEOMETRY[case["model"]]
        B, kind = case["batch"], case["kind"]
        ctx = fv.Context(hidden=heads * dh, heads=heads, head_dim=dh, ffn_hidden=4 * heads * dh, dtype=case["dtype"])
        first = second = ws = None
        if kind == "rope":
            first = fv.Rope(**_rope_settings(case))
        else:
            parts = [s[n] for n in ("k_codes", "v_codes", "k_scale", "v_scale")]
            if kind == "write" and case["ragged"]:
                first, second = fv.KVB(*parts, lens=s["first"]), fv.KVB(*parts, lens=s["last"])
            elif kind == "write":
                first, second = fv.KVB(*parts, len=case["prefix"]), fv.KVB(*parts, len=case["prefix"] + case["rows"])
            else:
                first = fv.KVB(*parts, len=case["keys"], lens=s["lens"], mask=s["mask"])
            size = 0
            if kind == "attend":
                size = fv.fvar_kvb_attention_workspace_bytes(ctx, first, B, case["queries"], case["weights"])
            elif kind == "evict":
                second = fv.KVB(s["to_k"], s["to_v"], s["to_k_scale"], s["to_v_scale"], lens=s["to_lens"])
                size = fv.fvar_kvb_evict_workspace_bytes(ctx, first, B, case["keep"])
            ws = torch.empty(size, dtype=torch.uint8, device="cuda")
        s["handle"] = (fv, ctx, first, second, ws)
    return s["handle"]


def _own(s):
    fv, ctx, first, second, ws = _handle(s)
    case = s["case"]
    B, kind = case["batch"], case["kind"]
    if kind == "rope":
        fv.fvar_rope_apply(ctx, first, s["pos"], B, case["rows"], s["q"], s["k"], s["q_out"], s["k_out"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if kind == "attend":
        fv.fvar_kvb_attention(ctx, s["q"], first, B, case["queries"], s["o"], ws, weights=s["weights"])
        return {"o": s["o"], "weights": s["weights"]} if case["weights"] else {"o": s["o"]}
    if kind == "write":
        fv.fvar_kvb_append(ctx, first, s["k"], s["v"], B, case["rows"])
        # the rows just written, and those before them that can share a block with the first
        rows = case["rows"] + BLOCK - 1
        fv.fvar_kvb_read(ctx, second, B, -rows, rows, s["k_back"], s["v_back"])
        return {"k": s["k_back"], "v": s["v_back"]}
    fv.fvar_kvb_evict(ctx, first, s["weights"], B, case["keep"], case["recent"], second, s["to_weights"], s["to_lens"], s["idx"], ws)
    fv.fvar_kvb_read(ctx, second, B, 0, case["keep"], s["k_back"], s["v_back"])
    return {"idx": s["idx"], "lens": s["to_lens"], "weights": s["to_weights"], "k": s["k_back"], "v": s["v_back"]}


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------ 64 bits
def _two(k):
    """2^k in 64 bits for tensors of whole numbers (a library's power may be off by the last bit)."""
    return ((k.long() + 1023) << 52).view(torch.float64)


def _held(codes, scales):
    """Values of codes [..., rows, dh] and scale bytes [..., rows]: sign, 4 bits of exponent, 3 of mantissa."""
    c = codes.long()
    expo, mant = (c // 8) % 16, (c % 8).double()
    mag = torch.where(expo == 0, mant / 512, (1 + mant / 8) * _two(expo - 7))
    mag = torch.where(c % 128 == 127, float("nan"), mag)
    return torch.where(c >= 128, -mag, mag) * _two(scales.long() - 127).unsqueeze(-1)


def _nearest(x, e):
    """Numbers x as the format holds them with the exponents e."""
    y = x / _two(e)
    step = _two(torch.frexp(y.abs().clamp_min(2.0 ** -6)).exponent - 4)
    return (torch.round(y / step) * step).clamp(-448, 448) * _two(e)


def _least(top):
    """The exponent of blocks whose largest numbers are `top`: 464 = .90625 * 2^9."""
    part, e = torch.frexp(top)
    return torch.where(top > 0, torch.where(part > 0.90625, e - 8, e - 9), -117).clamp(-117, 119)


def _exact_rope(s):
    case = s["case"]
    heads, dh = GEOMETRY[case["model"]]
    r = _rope_settings(case)
    P = r["dim"] // r["axes"]
    turns = []                                                     # per pair of one part
    for i in range(P // 2):
        if r["scaling"] == "ntk":
            turns.append((r["base"] * r["factor"] ** (P / (P - 2))) ** (-2 * i / P))
            continue
        f = r["base"] ** (-2 * i / P)
        if r["scaling"] == "linear":
            f /= r["factor"]
        elif r["scaling"] == "yarn":
            g = (r["original"] * f / (2 * math.pi) - r["low"]) / (r["high"] - r["low"])
            g = min(max(g, 0.0), 1.0)
            f = g * f + (1 - g) * f / r["factor"]
        turns.append(f)
    out = {}
    for name in ("q", "k"):
        x = s[name].double()
        y = x.clone()
        for a in range(r["axes"]):
            pos = (s["pos"][..., a] if r["axes"] == 2 else s["pos"]).double().unsqueeze(-1)
            for i in range(P // 2):
                one, two = (a * P + 2 * i, a * P + 2 * i + 1) if r["interleaved"] else (a * P + i, a * P + i + P // 2)
                w = torch.polar(torch.full_like(pos, r.get("magnitude", 1.0)), pos * turns[i])
                z = torch.complex(x[..., one], x[..., two]) * w
                y[..., one], y[..., two] = z.real, z.imag
        out[name] = y
    return out


def _exact_write(s):
    case = s["case"]
    out = {}
    for n in ("k", "v"):
        B, rows, hk, dh = s[n].shape
        back = torch.zeros((B, rows + BLOCK - 1, hk, dh), dtype=torch.float64, device="cuda")
        for b, first in enumerate(_lengths(case, case["prefix"])):
            start = first // BLOCK * BLOCK
            held = first - start
            old = _held(s[n + "_codes"][b, :, start:first], s[n + "_scale"][b, :, start // BLOCK].unsqueeze(-1).expand(hk, held))
            x = torch.cat([old, s[n][b].transpose(0, 1).double()], 1)
            x = torch.cat([x, x.new_zeros((hk, -x.shape[1] % BLOCK, dh))], 1).unflatten(1, (-1, BLOCK))
            y = x.clone()
            y[:, 0, :held] = 0
            e = _least(y.abs().amax((-2, -1)))
            if held:
                e[:, 0] = torch.maximum(e[:, 0], s[n + "_scale"][b, :, start // BLOCK].to(e.dtype) - 127)
            x = _nearest(x, e[..., None, None]).flatten(1, 2)[:, :held + rows]
            before = min(BLOCK - 1, first)                           # rows before the new ones that are read back
            if before > held:
                past = torch.arange(first - before, start, device="cuda")
                x = torch.cat([_held(s[n + "_codes"][b, :, past], s[n + "_scale"][b][:, past // BLOCK]), x], 1)
            elif before < held:
                x = x[:, held - before:]
            back[b, BLOCK - 1 - before:] = x.transpose(0, 1)
        out[n] = back
    return out


def _rows_of(s, n, b, j, pick):
    return _held(s[n + "_codes"][b, j, pick], s[n + "_scale"][b, j, pick // BLOCK])


def _exact_attend(s):
    case = s["case"]
    heads, dh = GEOMETRY[case["model"]]
    group = heads // case["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    got = torch.zeros((case["batch"], case["kv_heads"], case["keys"]), dtype=torch.float64, device="cuda")
    for b, length in enumerate(_lengths(case, case["keys"])):
        pick = torch.arange(length, device="cuda")
        if s["mask"] is not None:
            pick = pick[s["mask"][b, :length] != 0]
        if not pick.numel():
            continue
        for j in range(case["kv_heads"]):
            k, v = _rows_of(s, "k", b, j, pick), _rows_of(s, "v", b, j, pick)
            for h in range(j * group, (j + 1) * group):
                w = torch.softmax(s["q"][b, :, h].double() @ k.t().contiguous() / math.sqrt(dh), dim=-1)
                out[b, :, h] = w @ v
                got[b, j, pick] += w.sum(0)
    return {"o": out, "weights": got} if case["weights"] else {"o": out}


def _exact_evict(s):
    case = s["case"]
    _, dh = GEOMETRY[case["model"]]
    B, hk, keep = case["batch"], case["kv_heads"], case["keep"]
    out = {n: torch.zeros((B, keep, hk, dh), dtype=torch.float64, device="cuda") for n in ("k", "v")}
    idx = torch.full((B, hk, keep), -1, dtype=torch.int32, device="cuda")
    weights = torch.zeros((B, hk, keep), dtype=torch.float64, device="cuda")
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    for b, length in enumerate(_lengths(case, case["keys"])):
        pick = torch.arange(length, device="cuda")
        if s["mask"] is not None:
            pick = pick[s["mask"][b, :length] != 0]
        lens[b] = count = min(keep, pick.numel())
        late = pick[pick >= length - case["recent"]]
        early = pick[pick < length - case["recent"]]
        for j in range(hk if count else 0):
            best = torch.argsort(-s["weights"][b, j, early].double(), stable=True)[:count - late.numel()]
            rows = torch.cat([early[best].sort().values, late])
            idx[b, j, :count], weights[b, j, :count] = rows.to(torch.int32), s["weights"][b, j, rows].double()
            for n in ("k", "v"):
                x = _rows_of(s, n, b, j, rows)
                top = torch.nn.functional.pad(x.abs().amax(-1), (0, -count % BLOCK)).unflatten(0, (-1, BLOCK)).amax(-1)
                out[n][b, :count, j] = _nearest(x, _least(top).repeat_interleave(BLOCK)[:count].unsqueeze(-1))
    return dict(out, idx=idx, lens=lens, weights=weights)


def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "write": _exact_write, "attend": _exact_attend, "evict": _exact_evict}[case["kind"]](s)
