"""The operators of a key/value cache held in 4 bits, by which their speed and outputs are judged.

A program that generates images scale by scale keeps the keys and values of every scale.  Held in 4 bits they take
17/64 of the room of bf16.  Three things are done with such a cache: new rows are quantised into it as they are produced
("write", which also reads the new rows back), rows are read back ("read"), and queries attend over it ("attend").

Format: blocks of 32 consecutive elements of one token and head share a power of two 2^e, stored as the byte e + 127; an
element is one of 0, .5, 1, 1.5, 2, 3, 4, 6 and a sign (codes 0..7, 8 for the sign), element 2i in the low half of byte i.
e is the smallest integer for which max |x| < 7 * 2^e, within [-124, 125]; codes are the nearest values, ties to the even
code, and at most 6.
    codes  uint8 [batch, kv_heads, capacity, head_dim / 2]
    scales uint8 [batch, kv_heads, capacity, head_dim / 32]

Sizes are those of the workloads in `workloads/` (see perf/cases.py), with fewer kv heads than query heads as the generic
case; `draw` spreads over the same ranges, odd sizes included.
"""
from __future__ import annotations

import math

import torch

own = False

# heads, head_dim of the model shapes in `workloads/`
GEOMETRY = {"d1024": (16, 64), "d1920": (30, 64), "d2048": (16, 128), "d4096": (32, 128)}


def _write(model, kv_heads, batch, rows, prefix, dtype="bf16", ragged=False):
    return dict(kind="write", model=model, kv_heads=kv_heads, batch=batch, rows=rows, prefix=prefix, dtype=dtype,
                ragged=ragged)


def _read(model, kv_heads, batch, rows, dtype="bf16"):
    return dict(kind="read", model=model, kv_heads=kv_heads, batch=batch, rows=rows, dtype=dtype)


def _attend(model, kv_heads, batch, queries, keys, dtype="bf16", ragged=False, masked=False):
    return dict(kind="attend", model=model, kv_heads=kv_heads, batch=batch, queries=queries, keys=keys, dtype=dtype,
                ragged=ragged, masked=masked)


def listed():
    cases = {
        # one token of a single image behind the cache of all scales up to 64x64: latency
        "write_token_b1": _write("d2048", 16, 1, 1, 10520),
        # one token each of 32 sequences of different lengths, grouped heads: a serving step
        "write_tokens_b32": _write("d4096", 8, 32, 1, 16920, ragged=True),
        # 32-bit storage: the last scale (16x16) of the hidden-1024 model, two samples
        "write_f32": _write("d1024", 16, 2, 256, 424, dtype="f32"),
        # the largest shape: every token of the 80x80 scale, batch 4
        "write_large": _write("d4096", 32, 4, 6400, 10521),
        # the cache in front of the 24x24 scale at head_dim 64, odd number of rows
        "read_d64_b8": _read("d1920", 30, 8, 871),
        # the cache in front of the 40x40 scale of a serving batch
        "read_b32": _read("d2048", 16, 32, 2521),
        # one query of a single image over the whole cache: latency and the split of a long axis
        "attend_token_b1": _attend("d2048", 16, 1, 1, 10521),
        # one query each of 32 sequences of different lengths (one of them empty), grouped heads, some keys hidden
        "attend_tokens_b32": _attend("d4096", 8, 32, 1, 16921, ragged=True, masked=True),
        # the kept rows of the 24x24 scale at batch 8, head_dim 64
        "attend_d64_b8": _attend("d1920", 30, 8, 231, 871),
        # a serving batch: kept rows of the 40x40 scale, 16 images with guidance doubling
        "attend_b32": _attend("d2048", 16, 32, 480, 3001),
        # the largest shape: kept rows of the 80x80 scale over all earlier ones
        "attend_large": _attend("d4096", 32, 4, 1600, 12121),
        # 32-bit storage, a mask over the keys
        "attend_f32": _attend("d1024", 16, 2, 128, 552, dtype="f32", masked=True),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["write", "write", "read", "attend", "attend", "attend"])
    model = rng.choice(list(GEOMETRY))
    heads, dh = GEOMETRY[model]
    kv_heads = heads // rng.choice([g for g in (1, 1, 1, 2, 3, 4, 8) if heads % g == 0])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    batch = _log_int(rng, 1, 32)
    if kind != "attend":
        rows = _log_int(rng, 1, 6400)
        while batch * rows * kv_heads * dh > 5e7:                 # half the largest listed case's elements
            batch, rows = max(1, batch // 2), rows if batch > 1 else rows // 2
        if kind == "read":
            return _read(model, kv_heads, batch, rows, dtype)
        return _write(model, kv_heads, batch, rows, _log_int(rng, 1, 10521), dtype, rng.random() < 0.5)
    queries, keys = _log_int(rng, 1, 1600), _log_int(rng, 1, 16921)
    if dtype == "f32":
        queries, keys = min(queries, 256), max(1, keys // 8)
    while batch * heads * queries * keys > 1.2e9 or batch * kv_heads * keys * dh > 4e8:
        if batch > 1:
            batch //= 2
        else:
            queries, keys = max(1, queries * 3 // 4), max(1, keys * 3 // 4)
    return _attend(model, kv_heads, batch, queries, keys, dtype, rng.random() < 0.4, rng.random() < 0.3)


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
    codes = torch.empty((batch, heads, capacity, dh // 2), dtype=torch.uint8, device="cuda")
    scales = torch.empty((batch, heads, capacity, dh // 32), dtype=torch.uint8, device="cuda")
    for b in range(batch):
        codes[b], scales[b] = _quantise(_rows(g, 1, capacity, heads, dh, dt)[0].transpose(0, 1))
    return codes, scales


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    heads, dh = GEOMETRY[case["model"]]
    hk, B, dt = case["kv_heads"], case["batch"], _dtype(case)
    s = dict(case=case)

    def buf(*shape, dtype=dt):
        return torch.empty(shape, dtype=dtype, device="cuda")

    if case["kind"] == "write":
        capacity = case["prefix"] + case["rows"]
        for n in ("k", "v"):
            s[n] = _rows(g, B, case["rows"], hk, dh, dt).contiguous()
            s[n + "_codes"] = torch.zeros((B, hk, capacity, dh // 2), dtype=torch.uint8, device="cuda")
            s[n + "_scale"] = torch.zeros((B, hk, capacity, dh // 32), dtype=torch.uint8, device="cuda")
            s[n + "_back"] = buf(B, case["rows"], hk, dh)
        s["first"] = torch.tensor(_lengths(case, case["prefix"]), dtype=torch.int32, device="cuda")
        s["last"] = s["first"] + case["rows"]
        return s
    capacity = case["rows"] if case["kind"] == "read" else case["keys"]
    for n in ("k", "v"):
        s[n + "_codes"], s[n + "_scale"] = _cache(g, B, hk, capacity, dh, dt)
    if case["kind"] == "read":
        s.update(k_back=buf(B, capacity, hk, dh), v_back=buf(B, capacity, hk, dh))
        return s
    s["q"] = _randn(g, B, case["queries"], heads, dh).to(dt)
    s["o"] = buf(B, case["queries"], heads, dh)
    s["lens"] = torch.tensor(_lengths(case, capacity), dtype=torch.int32, device="cuda") if case["ragged"] else None
    s["mask"] = (torch.rand((B, capacity), generator=g, device="cuda") < 0.7).to(torch.uint8) if case["masked"] else None
    return s


def work(case):
    heads, dh = GEOMETRY[case["model"]]
    es = 2 if case["dtype"] == "bf16" else 4
    held = dh / 2 + dh / 32                                        # bytes of one row of one head
    if case["kind"] != "attend":
        rows = 2 * case["batch"] * case["rows"] * case["kv_heads"]     # K and V
        once = rows * (dh * es + held)
        return {"bytes": once * (2 if case["kind"] == "write" else 1), "flops": 0}
    keys = sum(_lengths(case, case["keys"]))
    seen = 0.7 * keys if case["masked"] else keys
    qo = 2 * case["batch"] * case["queries"] * heads * dh * es
    return {"bytes": qo + 2 * seen * case["kv_heads"] * held + (keys if case["masked"] else 0),
            "flops": 4.0 * seen * case["queries"] * heads * dh}


# ------------------------------------------------------------------------------------ plain form
def _power(e):
    """2^e for int32 tensors of exponents of normal numbers."""
    return ((e + 127) << 23).view(torch.float32)


def _quantise(x):
    """x [..., dh] -> codes [..., dh / 2], scales [..., dh / 32]."""
    x = x.float()
    x = x.reshape(*x.shape[:-1], -1, 32)
    top = x.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(top)                                        # top = m 2^e, m in [.5, 1)
    e = (e - 3 + (m >= 0.875).to(torch.int32)).clamp(-124, 125)
    e = torch.where(top == 0, -124, e)
    y = (x * _power(-e)).abs()
    code = ((y > 0.25).to(torch.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0))
    code = code + 8 * torch.signbit(x).to(torch.uint8)
    fine = torch.isfinite(top)
    code = torch.where(fine, code, 0).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), torch.where(fine, e + 127, 255).squeeze(-1).to(torch.uint8)


def _values(codes, scales):
    """The values that codes [..., dh / 2] and scales [..., dh / 32] stand for, in 32 bits."""
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0],
                         device=codes.device)
    code = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2)
    x = table[code.to(torch.int32)]
    scale = torch.where(scales == 255, float("nan"), _power(scales.to(torch.int32) - 127))
    return (x.reshape(*x.shape[:-1], -1, 32) * scale.unsqueeze(-1)).flatten(-2)


def _plain(s):
    case = s["case"]
    dt = _dtype(case)
    if case["kind"] == "read":
        return {n: _values(s[n + "_codes"], s[n + "_scale"]).transpose(1, 2).to(dt).contiguous() for n in ("k", "v")}
    if case["kind"] == "write":
        B, rows, hk = s["k"].shape[:3]
        at = (s["first"].long()[:, None, None] + torch.arange(rows, device="cuda")).expand(B, hk, rows).unsqueeze(-1)
        out = {}
        for n in ("k", "v"):
            held = (s[n + "_codes"], s[n + "_scale"])
            for buf, new in zip(held, _quantise(s[n].transpose(1, 2))):
                buf.scatter_(2, at.expand_as(new), new)
            back = [buf.gather(2, at.expand(B, hk, rows, buf.shape[-1])) for buf in held]
            out[n] = _values(*back).transpose(1, 2).to(dt).contiguous()
        return out
    heads, dh = GEOMETRY[case["model"]]
    B, n, hk, L = case["batch"], case["queries"], case["kv_heads"], case["keys"]
    k, v = _values(s["k_codes"], s["k_scale"]), _values(s["v_codes"], s["v_scale"])
    q = s["q"].float().reshape(B, n, hk, heads // hk, dh).permute(0, 2, 3, 1, 4).reshape(B, hk, -1, dh)
    x = torch.matmul(q, k.transpose(-1, -2).contiguous()) * dh ** -0.5
    if s["lens"] is not None or s["mask"] is not None:
        seen = torch.ones((B, L), dtype=torch.bool, device="cuda")
        if s["lens"] is not None:
            seen = seen & (torch.arange(L, device="cuda") < s["lens"][:, None])
        if s["mask"] is not None:
            seen = seen & (s["mask"] != 0)
        x = torch.where(seen[:, None, None], x, -math.inf)
        v = torch.where(seen[:, None, :, None], v, 0.0)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total == 0, 1.0, total)
    return o.reshape(B, hk, heads // hk, n, dh).permute(0, 3, 1, 2, 4).reshape(B, n, heads, dh).to(dt)


# ------------------------------------------------------------------------------------ the framework's own form
def _handle(s):
    """What a program keeps from call to call: the model's context, the cache's handle, the attention's workspace."""
    if "handle" not in s:
        import paper_2512_16483_amd as fv
        case = s["case"]
        heads, dh = GEOMETRY[case["model"]]
        ctx = fv.Context(hidden=heads * dh, heads=heads, head_dim=dh, ffn_hidden=4 * heads * dh, dtype=case["dtype"])
        parts = [s[n] for n in ("k_codes", "v_codes", "k_scale", "v_scale")]
        if case["kind"] == "write" and case["ragged"]:
            before, after = fv.KVQ(*parts, lens=s["first"]), fv.KVQ(*parts, lens=s["last"])
        elif case["kind"] == "write":
            before, after = fv.KVQ(*parts, len=case["prefix"]), fv.KVQ(*parts, len=case["prefix"] + case["rows"])
        elif case["kind"] == "read":
            before = after = fv.KVQ(*parts, len=case["rows"])
        else:
            before = after = fv.KVQ(*parts, len=case["keys"], lens=s["lens"], mask=s["mask"])
        ws = None
        if case["kind"] == "attend":
            ws = torch.empty(fv.fvar_kvq_attention_workspace_bytes(ctx, before, case["batch"], case["queries"]),
                             dtype=torch.uint8, device="cuda")
        s["handle"] = (fv, ctx, before, after, ws)
    return s["handle"]


def _own(s):
    fv, ctx, before, after, ws = _handle(s)
    case = s["case"]
    B = case["batch"]
    if case["kind"] == "attend":
        fv.fvar_kvq_attention(ctx, s["q"], before, B, case["queries"], s["o"], ws)
        return s["o"]
    if case["kind"] == "write":
        fv.fvar_kvq_append(ctx, before, s["k"], s["v"], B, case["rows"])
        # the rows just written: the last `rows` of every sample
        fv.fvar_kvq_read(ctx, after, B, -case["rows"], case["rows"], s["k_back"], s["v_back"])
    else:
        fv.fvar_kvq_read(ctx, after, B, 0, case["rows"], s["k_back"], s["v_back"])
    return {"k": s["k_back"], "v": s["v_back"]}


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------ 64 bits
def _nearest(x):
    """Rows x [..., dh] as the format holds them, by its definition."""
    blocks = x.double().unflatten(-1, (-1, 32))
    top = blocks.abs().amax(-1, keepdim=True)
    e = torch.where(top > 0, torch.floor(torch.log2(top / 7)) + 1, -124.0).clamp(-124, 125)
    y = blocks / 2.0 ** e
    binade = torch.floor(torch.log2(y.abs().clamp_min(0.25))).clamp_min(0.0)
    step = 2.0 ** (binade - 1)
    return ((torch.round(y / step) * step).clamp(-6, 6) * 2.0 ** e).flatten(-2)


def _held(codes, scales):
    """Values of codes and scales: sign, 2-bit exponent, 1-bit mantissa."""
    c = torch.stack([codes % 16, codes // 16], -1).flatten(-2).long()
    expo, mant = (c // 2) % 4, (c % 2).double()
    mag = torch.where(expo == 0, 0.5 * mant, (1 + 0.5 * mant) * 2.0 ** (expo - 1).double())
    size = 2.0 ** (scales.double() - 127)
    return torch.where(c >= 8, -mag, mag) * size.repeat_interleave(32, dim=-1)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "write":
        return {n: _nearest(s[n]) for n in ("k", "v")}
    if case["kind"] == "read":
        return {n: _held(s[n + "_codes"], s[n + "_scale"]).transpose(1, 2) for n in ("k", "v")}
    heads, dh = GEOMETRY[case["model"]]
    group = heads // case["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for b, length in enumerate(_lengths(case, case["keys"])):
        pick = torch.arange(length, device="cuda")
        if s["mask"] is not None:
            pick = pick[s["mask"][b, :length] != 0]
        if not pick.numel():
            continue
        for j in range(case["kv_heads"]):
            k, v = (_held(s[n + "_codes"][b, j, pick], s[n + "_scale"][b, j, pick]) for n in ("k", "v"))
            for h in range(j * group, (j + 1) * group):
                w = torch.softmax(s["q"][b, :, h].double() @ k.t().contiguous() / math.sqrt(dh), dim=-1)
                out[b, :, h] = w @ v
    return out
