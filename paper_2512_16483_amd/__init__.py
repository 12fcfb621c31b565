"""Python binding of libfvar.so (argument marshalling only; all compute is in the HIP kernels).

The functions carry the names of the C entry points in include/fvar.h and take torch tensors
that live on the GPU; PyTorch is used for device memory and streams only.  Loading fails loudly
when the library has not been built (python -m paper_2512_16483_amd.build)."""
from __future__ import annotations

import ctypes as C
import math
import os
from typing import Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfvar.so")

FVAR_OK, FVAR_ERR_INVALID_ARG, FVAR_ERR_UNSUPPORTED, FVAR_ERR_WORKSPACE, FVAR_ERR_HIP = range(5)
FVAR_F32, FVAR_BF16 = 0, 1

EXPORTS = (
    "fvar_create", "fvar_destroy", "fvar_last_error", "fvar_status_string", "fvar_keep_count",
    "fvar_scale_tokens", "fvar_scale_prev_len", "fvar_select_workspace_bytes",
    "fvar_block_workspace_bytes", "fvar_score_select", "fvar_block_forward_dense",
    "fvar_block_forward_pruned", "fvar_lowrank_fill", "fvar_rp_project", "fvar_cache_fill",
    "fvar_factors_workspace_bytes", "fvar_cache_factors", "fvar_upsample_tokens",
    "fvar_profile_enable",
    "fvar_profile_read", "fvar_debug_checks", "fvar_score_select_static",
    "fvar_fill_scored_workspace_bytes", "fvar_lowrank_fill_scored",
    "fvar_kvq_append", "fvar_kvq_read", "fvar_kvq_attention_workspace_bytes", "fvar_kvq_attention",
    "fvar_block_kvq_workspace_bytes", "fvar_block_forward_dense_kvq", "fvar_block_forward_pruned_kvq",
    "fvar_rope_init", "fvar_rope_apply", "fvar_kvb_append", "fvar_kvb_read", "fvar_kvb_attention_workspace_bytes",
    "fvar_kvb_attention", "fvar_kvb_evict_workspace_bytes", "fvar_kvb_evict",
    "fvar_block_kvb_workspace_bytes", "fvar_block_forward_dense_kvb", "fvar_block_forward_pruned_kvb",
)


class FvarError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"fvar status {status}: {msg}")
        self.status = status


class _Config(C.Structure):
    _fields_ = [("hidden", C.c_int32), ("heads", C.c_int32), ("head_dim", C.c_int32),
                ("ffn_hidden", C.c_int32), ("num_scales", C.c_int32),
                ("scale_hw", C.POINTER(C.c_int32)), ("dtype", C.c_int), ("ln_eps", C.c_float),
                ("attn_scale", C.c_float)]


class _Weights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in (
        "ln1_g", "ln1_b", "w_qkv", "b_qkv", "w_o", "b_o", "ln2_g", "ln2_b",
        "w_fc1", "b_fc1", "w_fc2", "b_fc2")]


class _KV(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("capacity", C.c_int32), ("len", C.c_int32)]


class _KVQ(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("lens", C.c_void_p), ("mask", C.c_void_p), ("kv_heads", C.c_int32), ("capacity", C.c_int32),
                ("len", C.c_int32)]


class _KVB(C.Structure):
    _fields_ = _KVQ._fields_


class _Rope(C.Structure):
    _fields_ = [("dim", C.c_int32), ("axes", C.c_int32), ("interleaved", C.c_int32), ("scaling", C.c_int32), ("base", C.c_double),
                ("factor", C.c_double), ("original", C.c_double), ("low", C.c_double), ("high", C.c_double), ("magnitude", C.c_double),
                ("turns", C.c_double * 64)]


class _ProfileEntry(C.Structure):
    _fields_ = [("label", C.c_char * 48), ("launches", C.c_int64), ("total_ms", C.c_double)]


_lib = None


def load_library() -> C.CDLL:
    """dlopen libfvar.so and declare the prototypes; raises if it is not built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with "
                          "`python -m paper_2512_16483_amd.build` (there is no fallback path)")
    lib = C.CDLL(LIB_PATH)
    vp, i32, sz = C.c_void_p, C.c_int32, C.c_size_t
    lib.fvar_create.argtypes = [C.POINTER(_Config), C.POINTER(vp)]
    lib.fvar_create.restype = C.c_int
    lib.fvar_destroy.argtypes = [vp]
    lib.fvar_destroy.restype = None
    lib.fvar_last_error.argtypes = [vp]
    lib.fvar_last_error.restype = C.c_char_p
    lib.fvar_status_string.argtypes = [C.c_int]
    lib.fvar_status_string.restype = C.c_char_p
    lib.fvar_keep_count.argtypes = [i32, i32, i32]
    lib.fvar_keep_count.restype = i32
    lib.fvar_scale_tokens.argtypes = [vp, i32]
    lib.fvar_scale_tokens.restype = i32
    lib.fvar_scale_prev_len.argtypes = [vp, i32]
    lib.fvar_scale_prev_len.restype = i32
    lib.fvar_select_workspace_bytes.argtypes = [vp, i32, i32]
    lib.fvar_select_workspace_bytes.restype = sz
    lib.fvar_block_workspace_bytes.argtypes = [vp, i32, i32]
    lib.fvar_block_workspace_bytes.restype = sz
    lib.fvar_score_select.argtypes = [vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, vp, sz]
    lib.fvar_score_select.restype = C.c_int
    lib.fvar_block_forward_dense.argtypes = [vp, vp, C.POINTER(_Weights), vp, i32, i32,
                                             C.POINTER(_KV), vp, vp, sz]
    lib.fvar_block_forward_dense.restype = C.c_int
    lib.fvar_block_forward_pruned.argtypes = [vp, vp, C.POINTER(_Weights), vp, i32, i32, vp, i32,
                                              C.POINTER(_KV), vp, vp, sz]
    lib.fvar_block_forward_pruned.restype = C.c_int
    lib.fvar_lowrank_fill.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, vp, vp, vp]
    lib.fvar_lowrank_fill.restype = C.c_int
    lib.fvar_fill_scored_workspace_bytes.argtypes = [vp, i32, i32]
    lib.fvar_fill_scored_workspace_bytes.restype = sz
    lib.fvar_lowrank_fill_scored.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, vp, vp, vp, vp, vp, sz]
    lib.fvar_lowrank_fill_scored.restype = C.c_int
    lib.fvar_rp_project.argtypes = [vp, vp, vp, i32, vp, i32, i32, i32, vp]
    lib.fvar_rp_project.restype = C.c_int
    lib.fvar_cache_fill.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, vp, vp]
    lib.fvar_cache_fill.restype = C.c_int
    lib.fvar_factors_workspace_bytes.argtypes = [vp, i32, i32, i32]
    lib.fvar_factors_workspace_bytes.restype = sz
    lib.fvar_cache_factors.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, C.c_double, vp, vp, vp, sz]
    lib.fvar_cache_factors.restype = C.c_int
    lib.fvar_upsample_tokens.argtypes = [vp, vp, vp, i32, i32, i32, i32, i32, i32, vp]
    lib.fvar_upsample_tokens.restype = C.c_int
    lib.fvar_score_select_static.argtypes = [vp, vp, vp, i32, i32, i32, vp, vp]
    lib.fvar_score_select_static.restype = C.c_int
    lib.fvar_debug_checks.argtypes = [vp, i32]
    lib.fvar_debug_checks.restype = C.c_int
    kvq = C.POINTER(_KVQ)
    lib.fvar_kvq_append.argtypes = [vp, vp, kvq, vp, vp, i32, i32, i32]
    lib.fvar_kvq_append.restype = C.c_int
    lib.fvar_kvq_read.argtypes = [vp, vp, kvq, i32, i32, i32, vp, vp]
    lib.fvar_kvq_read.restype = C.c_int
    lib.fvar_kvq_attention_workspace_bytes.argtypes = [vp, kvq, i32, i32]
    lib.fvar_kvq_attention_workspace_bytes.restype = sz
    lib.fvar_kvq_attention.argtypes = [vp, vp, vp, i32, kvq, i32, i32, vp, vp, sz]
    lib.fvar_kvq_attention.restype = C.c_int
    lib.fvar_block_kvq_workspace_bytes.argtypes = [vp, kvq, i32, i32]
    lib.fvar_block_kvq_workspace_bytes.restype = sz
    lib.fvar_block_forward_dense_kvq.argtypes = [vp, vp, C.POINTER(_Weights), vp, i32, i32, kvq, vp, vp, sz]
    lib.fvar_block_forward_dense_kvq.restype = C.c_int
    lib.fvar_block_forward_pruned_kvq.argtypes = [vp, vp, C.POINTER(_Weights), vp, i32, i32, vp, i32, kvq, vp, vp, sz]
    lib.fvar_block_forward_pruned_kvq.restype = C.c_int
    rope, kvb = C.POINTER(_Rope), C.POINTER(_KVB)
    lib.fvar_rope_init.argtypes = [rope]
    lib.fvar_rope_init.restype = C.c_int
    lib.fvar_rope_apply.argtypes = [vp, vp, rope, vp, i32, i32, i32, vp, i32, vp, i32, vp, i32, vp, i32]
    lib.fvar_rope_apply.restype = C.c_int
    lib.fvar_kvb_append.argtypes = [vp, vp, kvb, vp, vp, i32, i32, i32]
    lib.fvar_kvb_append.restype = C.c_int
    lib.fvar_kvb_read.argtypes = [vp, vp, kvb, i32, i32, i32, vp, vp]
    lib.fvar_kvb_read.restype = C.c_int
    lib.fvar_kvb_attention_workspace_bytes.argtypes = [vp, kvb, i32, i32, i32]
    lib.fvar_kvb_attention_workspace_bytes.restype = sz
    lib.fvar_kvb_attention.argtypes = [vp, vp, vp, i32, kvb, i32, i32, vp, vp, i32, vp, sz]
    lib.fvar_kvb_attention.restype = C.c_int
    lib.fvar_kvb_evict_workspace_bytes.argtypes = [vp, kvb, i32, i32]
    lib.fvar_kvb_evict_workspace_bytes.restype = sz
    lib.fvar_kvb_evict.argtypes = [vp, vp, kvb, vp, i32, i32, i32, kvb, vp, vp, vp, vp, sz]
    lib.fvar_kvb_evict.restype = C.c_int
    lib.fvar_block_kvb_workspace_bytes.argtypes = [vp, kvb, i32, i32, i32]
    lib.fvar_block_kvb_workspace_bytes.restype = sz
    lib.fvar_block_forward_dense_kvb.argtypes = [vp, vp, C.POINTER(_Weights), vp, i32, i32, kvb, rope, vp, vp, i32, vp, vp, sz]
    lib.fvar_block_forward_dense_kvb.restype = C.c_int
    lib.fvar_block_forward_pruned_kvb.argtypes = [vp, vp, C.POINTER(_Weights), vp, i32, i32, vp, i32, kvb, rope, vp, vp, i32, vp, vp, sz]
    lib.fvar_block_forward_pruned_kvb.restype = C.c_int
    lib.fvar_profile_enable.argtypes = [vp, i32]
    lib.fvar_profile_enable.restype = C.c_int
    lib.fvar_profile_read.argtypes = [vp, C.POINTER(_ProfileEntry), i32]
    lib.fvar_profile_read.restype = i32
    _lib = lib
    return lib


def _ptr(t) -> Optional[int]:
    """Device pointer of a contiguous torch tensor (None passes NULL)."""
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("tensors handed to fvar must be contiguous GPU tensors")
    return t.data_ptr()


def _nbytes(t) -> int:
    return 0 if t is None else t.numel() * t.element_size()


_current: list = []                                           # what gives the current stream of a device, and that device


def _stream(stream) -> Optional[int]:
    if stream is None:
        if not _current:
            import torch
            raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)   # a Stream object takes 3 us, as long as a launch
            _current.append((raw, torch.cuda.current_device) if raw is not None else (torch.cuda.current_stream, lambda: None))
        of, device = _current[0]
        stream = of(device())
    return getattr(stream, "cuda_stream", stream) or None


class Context:
    """Owns one fvar_ctx."""

    def __init__(self, hidden: int, heads: int, head_dim: int, ffn_hidden: int,
                 scales: Sequence[int] = (), dtype: str = "bf16", ln_eps: float = 0.0,
                 attn_scale: float = 0.0):
        self.lib = load_library()
        hw = []
        for s in scales:
            hw += list(s) if isinstance(s, (tuple, list)) else [s, s]
        arr = (C.c_int32 * max(len(hw), 1))(*hw)
        cfg = _Config(hidden, heads, head_dim, ffn_hidden, len(hw) // 2, arr,
                      {"f32": FVAR_F32, "bf16": FVAR_BF16}[dtype], ln_eps, attn_scale)
        h = C.c_void_p()
        st = self.lib.fvar_create(C.byref(cfg), C.byref(h))
        if st != FVAR_OK:
            raise FvarError(st, "fvar_create: " + self.lib.fvar_status_string(st).decode())
        self.handle = h
        self.hidden, self.heads, self.head_dim, self.ffn_hidden = hidden, heads, head_dim, ffn_hidden
        self.dtype = dtype

    def check(self, st: int) -> None:
        if st != FVAR_OK:
            raise FvarError(st, self.lib.fvar_last_error(self.handle).decode())

    def close(self) -> None:
        if getattr(self, "handle", None):
            self.lib.fvar_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def fvar_create(**kw) -> Context:
    return Context(**kw)


def fvar_destroy(ctx: Context) -> None:
    ctx.close()


def fvar_keep_count(M: int, keep_num: int, keep_den: int) -> int:
    return load_library().fvar_keep_count(M, keep_num, keep_den)


def fvar_scale_tokens(ctx: Context, scale_index: int) -> int:
    return ctx.lib.fvar_scale_tokens(ctx.handle, scale_index)


def fvar_scale_prev_len(ctx: Context, scale_index: int) -> int:
    return ctx.lib.fvar_scale_prev_len(ctx.handle, scale_index)


def fvar_select_workspace_bytes(ctx: Context, B: int, M: int) -> int:
    return ctx.lib.fvar_select_workspace_bytes(ctx.handle, B, M)


def fvar_block_workspace_bytes(ctx: Context, B: int, rows: int) -> int:
    return ctx.lib.fvar_block_workspace_bytes(ctx.handle, B, rows)


def fvar_score_select(ctx: Context, x, B: int, M: int, k: int, idx_keep, idx_drop=None,
                      scores_in=None, scores_out=None, ws=None, stream=None) -> None:
    ctx.check(ctx.lib.fvar_score_select(ctx.handle, _stream(stream), _ptr(x), B, M, k,
                                        _ptr(scores_in), _ptr(scores_out), _ptr(idx_keep),
                                        _ptr(idx_drop), _ptr(ws), _nbytes(ws)))


def fvar_score_select_static(ctx: Context, x, B: int, M: int, k: int, idx_keep, idx_drop=None,
                             stream=None) -> None:
    ctx.check(ctx.lib.fvar_score_select_static(ctx.handle, _stream(stream), _ptr(x), B, M, k,
                                               _ptr(idx_keep), _ptr(idx_drop)))


def fvar_debug_checks(ctx: Context, on: bool) -> None:
    ctx.check(ctx.lib.fvar_debug_checks(ctx.handle, 1 if on else 0))


def _weights(w: dict) -> _Weights:
    s = _Weights()
    for name, _ in _Weights._fields_:
        setattr(s, name, _ptr(w.get(name)))
    return s


def fvar_block_forward_dense(ctx: Context, w: dict, x, B: int, M: int, kv_k, kv_v, capacity: int,
                             kv_len: int, y, ws, stream=None) -> None:
    kv = _KV(_ptr(kv_k), _ptr(kv_v), capacity, kv_len)
    ws_ = _weights(w)
    ctx.check(ctx.lib.fvar_block_forward_dense(ctx.handle, _stream(stream), C.byref(ws_), _ptr(x),
                                               B, M, C.byref(kv), _ptr(y), _ptr(ws), _nbytes(ws)))


def fvar_block_forward_pruned(ctx: Context, w: dict, x, B: int, M: int, idx_keep, k: int, kv_k,
                              kv_v, capacity: int, kv_len: int, y_keep, ws, stream=None) -> None:
    kv = _KV(_ptr(kv_k), _ptr(kv_v), capacity, kv_len)
    ws_ = _weights(w)
    ctx.check(ctx.lib.fvar_block_forward_pruned(ctx.handle, _stream(stream), C.byref(ws_), _ptr(x),
                                                B, M, _ptr(idx_keep), k, C.byref(kv), _ptr(y_keep),
                                                _ptr(ws), _nbytes(ws)))


def fvar_lowrank_fill(ctx: Context, y_keep, idx_keep, idx_drop, B: int, M: int, k: int, r: int,
                      w_c, g_c, y, stream=None) -> None:
    ctx.check(ctx.lib.fvar_lowrank_fill(ctx.handle, _stream(stream), _ptr(y_keep), _ptr(idx_keep),
                                        _ptr(idx_drop), B, M, k, r, _ptr(w_c), _ptr(g_c), _ptr(y)))


def fvar_fill_scored_workspace_bytes(ctx: Context, B: int, M: int) -> int:
    return ctx.lib.fvar_fill_scored_workspace_bytes(ctx.handle, B, M)


def fvar_lowrank_fill_scored(ctx: Context, y_keep, idx_keep, idx_drop, B: int, M: int, k: int, r: int,
                             w_c, g_c, y, scores_out, ws, stream=None) -> None:
    ctx.check(ctx.lib.fvar_lowrank_fill_scored(ctx.handle, _stream(stream), _ptr(y_keep),
                                               _ptr(idx_keep), _ptr(idx_drop), B, M, k, r, _ptr(w_c),
                                               _ptr(g_c), _ptr(y), _ptr(scores_out), _ptr(ws),
                                               _nbytes(ws)))


def fvar_rp_project(ctx: Context, qt, q_per_sample: bool, x, B: int, M: int, rows: int, out,
                    stream=None) -> None:
    ctx.check(ctx.lib.fvar_rp_project(ctx.handle, _stream(stream), _ptr(qt), 1 if q_per_sample else 0,
                                      _ptr(x), B, M, rows, _ptr(out)))


def fvar_cache_fill(ctx: Context, y_keep, idx_keep, idx_drop, B: int, M: int, k: int, cache, y,
                    stream=None) -> None:
    ctx.check(ctx.lib.fvar_cache_fill(ctx.handle, _stream(stream), _ptr(y_keep), _ptr(idx_keep),
                                      _ptr(idx_drop), B, M, k, _ptr(cache), _ptr(y)))


def fvar_factors_workspace_bytes(ctx: Context, B: int, M: int, r: int) -> int:
    return ctx.lib.fvar_factors_workspace_bytes(ctx.handle, B, M, r)


def fvar_cache_factors(ctx: Context, cache, qt, q_per_sample: bool, B: int, M: int, r: int,
                       ridge: float, w_c, g_c, ws, stream=None) -> None:
    ctx.check(ctx.lib.fvar_cache_factors(ctx.handle, _stream(stream), _ptr(cache), _ptr(qt),
                                         1 if q_per_sample else 0, B, M, r, float(ridge), _ptr(w_c),
                                         _ptr(g_c), _ptr(ws), _nbytes(ws)))


def fvar_upsample_tokens(ctx: Context, src, B: int, hs: int, ws: int, c: int, hd: int, wd: int, dst,
                         stream=None) -> None:
    ctx.check(ctx.lib.fvar_upsample_tokens(ctx.handle, _stream(stream), _ptr(src), B, hs, ws, c, hd,
                                           wd, _ptr(dst)))


class _Cache:
    """What KVQ and KVB have in common: the tensors of a cache, which its C structure points to, and the rows that it holds."""

    def _set_up(self, c, shapes: dict, head_dim: int, tensors: dict) -> None:
        self._shapes, self._tensors = shapes, {}
        self._c = c
        self._ref, self._batch, self._head_dim = C.byref(c), shapes["lens"][0], head_dim
        for name, t in tensors.items():
            self._hold(name, t)

    def _hold(self, name: str, t) -> None:
        """Tensor and pointer change together: the calls read what the attribute shows, and it lives as long."""
        if t is not None:
            if tuple(t.shape) != self._shapes[name]:
                raise ValueError(f"{name} has shape {tuple(t.shape)}, {self._shapes[name]} is wanted")
            kinds = ("torch.int32",) if name == "lens" else ("torch.uint8", "torch.bool") if name == "mask" else ("torch.uint8",)
            if str(t.dtype) not in kinds:
                raise ValueError(f"{name} is {t.dtype}, {' or '.join(kinds)} is wanted")
        elif name not in ("lens", "mask"):
            raise ValueError(f"{name} is None")
        setattr(self._c, name, _ptr(t))
        self._tensors[name] = t

    k = property(lambda self: self._tensors["k"], lambda self, t: self._hold("k", t))
    v = property(lambda self: self._tensors["v"], lambda self, t: self._hold("v", t))
    k_scale = property(lambda self: self._tensors["k_scale"], lambda self, t: self._hold("k_scale", t))
    v_scale = property(lambda self: self._tensors["v_scale"], lambda self, t: self._hold("v_scale", t))
    lens = property(lambda self: self._tensors["lens"], lambda self, t: self._hold("lens", t))
    mask = property(lambda self: self._tensors["mask"], lambda self, t: self._hold("mask", t))
    kv_heads = property(lambda self: self._c.kv_heads)
    capacity = property(lambda self: self._c.capacity)
    batch = property(lambda self: self._batch)
    head_dim = property(lambda self: self._head_dim)

    @property
    def len(self) -> int:
        return self._c.len

    @len.setter
    def len(self, value: int) -> None:
        self._c.len = value

    def _for(self, ctx: Context, B: int):
        if self._head_dim != ctx.head_dim or B > self._batch:
            raise ValueError(f"a cache of {self.batch} samples with head_dim {self.head_dim} does not serve {B} samples "
                             f"with head_dim {ctx.head_dim}")
        return self._ref


class KVQ(_Cache):
    """Key/value cache of one block in 4 bits: the tensors of fvar_kvq and the rows that it holds.

    k, v: uint8 [B, kv_heads, capacity, head_dim / 2]; k_scale, v_scale: uint8 [B, kv_heads, capacity, head_dim / 32];
    lens: int32 [B] on the GPU, or None where every sample holds `len` rows; mask: uint8 or bool [B, capacity], 0 hides a
    row from the attention, or None.  The tensors and `len` may be assigned to, tensors of the same shape; they are the caller's,
    who advances len or lens."""

    def __init__(self, k, v, k_scale, v_scale, len: int = 0, lens=None, mask=None):
        B, heads, capacity, codes = k.shape
        held, scales = (B, heads, capacity, codes), (B, heads, capacity, codes // 16)
        self._set_up(_KVQ(kv_heads=heads, capacity=capacity, len=len),
                     {"k": held, "v": held, "k_scale": scales, "v_scale": scales, "lens": (B,), "mask": (B, capacity)}, 2 * codes,
                     {"k": k, "v": v, "k_scale": k_scale, "v_scale": v_scale, "lens": lens, "mask": mask})


class KVB(_Cache):
    """Key/value cache of one block in 8 bits: the tensors of fvar_kvb and the rows that it holds, as KVQ but for
    k, v: uint8 [B, kv_heads, capacity, head_dim]; k_scale, v_scale: uint8 [B, kv_heads, ceil(capacity / 32)]."""

    def __init__(self, k, v, k_scale, v_scale, len: int = 0, lens=None, mask=None):
        B, heads, capacity, head_dim = k.shape
        held, scales = (B, heads, capacity, head_dim), (B, heads, (capacity + 31) // 32)
        self._set_up(_KVB(kv_heads=heads, capacity=capacity, len=len),
                     {"k": held, "v": held, "k_scale": scales, "v_scale": scales, "lens": (B,), "mask": (B, capacity)}, head_dim,
                     {"k": k, "v": v, "k_scale": k_scale, "v_scale": v_scale, "lens": lens, "mask": mask})


_KINDS: dict = {}                                             # element types by the contexts' names for them


def _kind(name: str):
    if not _KINDS:
        import torch
        _KINDS.update(bf16=torch.bfloat16, f32=torch.float32, i32=torch.int32)
    return _KINDS[name]


def _check_room(t, B: int, rows: int, width: int) -> None:
    """A contiguous tensor that has not just the elements of [B, rows, width]: it may have more where those are its first ones, in a flat one,
    in rows of `width`, in more samples, or in more rows of the only one."""
    n, s = t.numel(), t.shape if width > 1 else (*t.shape, 1)
    fits = n > B * rows * width and (len(s) == 1 or s[-1] == width and len(s) == 2 or
                                     len(s) > 2 and s[0] * s[1] * width == n and (s[1] == rows or B == 1 and s[1] > rows))
    if not fits:
        raise ValueError(f"{B} x {rows} rows of {width} elements are wanted, got a tensor of shape {tuple(t.shape)}")


def _packed(t, kind, B: int, rows: int, width: int) -> Optional[int]:
    """Pointer of contiguous t:[B, rows, width], whose type and size are looked at (None passes NULL)."""
    if t is None:
        return None
    if t.dtype is not kind:
        raise ValueError(f"a tensor of {kind} is wanted, got {t.dtype}")
    if not t.is_cuda or not t.is_contiguous():
        return _ptr(t)                                        # (which says what is wrong)
    if t.numel() != B * rows * width:
        _check_room(t, B, rows, width)
    return t.data_ptr()


def _rows(t, kind, B: int, rows: int, width: int):
    """Pointer and row pitch of t:[B, rows, ...] of the context's type, whose rows of `width` elements are contiguous; they may lie apart,
    as the parts of a fused projection's output do."""
    if t is None or t.is_contiguous():
        return _packed(t, kind, B, rows, width), 0
    if not t.is_cuda or t.dtype is not kind:
        raise ValueError(f"tensors handed to fvar must be GPU tensors, here of {kind}")
    shape, strides, run = t.shape, t.stride(), 1
    for i in range(len(shape) - 1, 1, -1):                    # (a view of a row, to ask it, takes longer than a launch)
        if shape[i] != 1 and strides[i] != run:
            run = -1
            break
        run *= shape[i]
    if len(shape) < 3 or shape[0] != B or shape[1] != rows or run != width:
        raise ValueError(f"[{B}, {rows}, ...] with contiguous rows of {width} elements is wanted, got shape "
                         f"{tuple(shape)} with strides {strides}")
    ld = strides[1] if rows > 1 else strides[0]
    if ld < width:                                            # rows that share memory, or one broadcast over them: 0 would mean packed
        raise ValueError(f"rows of {width} elements cannot be {ld} elements apart: a copy of the tensor is wanted")
    if B > 1 and strides[0] != rows * ld:
        raise ValueError("the rows of all samples have to be equally far apart")
    return t.data_ptr(), ld


def fvar_kvq_append(ctx: Context, kv: KVQ, k, v, B: int, rows: int, stream=None) -> None:
    kind, width = _kind(ctx.dtype), kv._c.kv_heads * ctx.head_dim
    (kp, ldk), (vp, ldv) = _rows(k, kind, B, rows, width), _rows(v, kind, B, rows, width)
    if (ldk or width) != (ldv or width):
        raise ValueError("k and v have different distances between rows")
    ctx.check(ctx.lib.fvar_kvq_append(ctx.handle, _stream(stream), kv._for(ctx, B), kp, vp, ldk, B, rows))


def fvar_kvq_read(ctx: Context, kv: KVQ, B: int, first: int, rows: int, k=None, v=None, stream=None) -> None:
    kind, width = _kind(ctx.dtype), kv._c.kv_heads * ctx.head_dim
    kp, vp = _packed(k, kind, B, rows, width), _packed(v, kind, B, rows, width)
    ctx.check(ctx.lib.fvar_kvq_read(ctx.handle, _stream(stream), kv._for(ctx, B), B, first, rows, kp, vp))


def fvar_kvq_attention_workspace_bytes(ctx: Context, kv: KVQ, B: int, n: int) -> int:
    return ctx.lib.fvar_kvq_attention_workspace_bytes(ctx.handle, kv._for(ctx, B), B, n)


def fvar_kvq_attention(ctx: Context, q, kv: KVQ, B: int, n: int, o, ws=None, stream=None) -> None:
    kind = _kind(ctx.dtype)
    qp, ld = _rows(q, kind, B, n, ctx.hidden)
    op = _packed(o, kind, B, n, ctx.hidden)
    ctx.check(ctx.lib.fvar_kvq_attention(ctx.handle, _stream(stream), qp, ld, kv._for(ctx, B), B, n, op, _ptr(ws), _nbytes(ws)))


def fvar_block_kvq_workspace_bytes(ctx: Context, kv: KVQ, B: int, rows: int) -> int:
    return ctx.lib.fvar_block_kvq_workspace_bytes(ctx.handle, kv._for(ctx, B), B, rows)


def fvar_block_forward_dense_kvq(ctx: Context, w: dict, x, B: int, M: int, kv: KVQ, y, ws, stream=None) -> None:
    ws_, kind = _weights(w), _kind(ctx.dtype)
    xp, yp = _packed(x, kind, B, M, ctx.hidden), _packed(y, kind, B, M, ctx.hidden)
    ctx.check(ctx.lib.fvar_block_forward_dense_kvq(ctx.handle, _stream(stream), C.byref(ws_), xp, B, M, kv._for(ctx, B), yp, _ptr(ws),
                                                   _nbytes(ws)))


def fvar_block_forward_pruned_kvq(ctx: Context, w: dict, x, B: int, M: int, idx_keep, k: int, kv: KVQ, y_keep, ws,
                                  stream=None) -> None:
    ws_, kind = _weights(w), _kind(ctx.dtype)
    xp, yp = _packed(x, kind, B, M, ctx.hidden), _packed(y_keep, kind, B, k, ctx.hidden)
    ctx.check(ctx.lib.fvar_block_forward_pruned_kvq(ctx.handle, _stream(stream), C.byref(ws_), xp, B, M,
                                                    _packed(idx_keep, _kind("i32"), B, k, 1), k, kv._for(ctx, B), yp, _ptr(ws),
                                                    _nbytes(ws)))


class Rope:
    """Rotary positions of a model, see fvar_rope.  scaling: "none", "linear", "ntk" or "yarn"; turns: frequencies of the caller's own, in
    turns per position, for each pair of a part."""

    def __init__(self, dim: int, interleaved: bool = False, axes: int = 1, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                 original: float = 0.0, low: float = 1.0, high: float = 32.0, magnitude: float = 0.0, turns: Optional[Sequence[float]] = None):
        self._c = _Rope(dim, axes, 1 if interleaved else 0, {"none": 0, "linear": 1, "ntk": 2, "yarn": 3}[scaling], base, factor, original,
                        low, high, magnitude)
        st = load_library().fvar_rope_init(C.byref(self._c))
        if st != FVAR_OK:
            raise FvarError(st, "fvar_rope_init: " + load_library().fvar_status_string(st).decode())
        if turns is not None:
            if len(turns) != dim // axes // 2:
                raise ValueError(f"{dim // axes // 2} frequencies are wanted, got {len(turns)}")
            if not all(math.isfinite(t) for t in turns):
                raise ValueError("frequencies have to be finite")
            self._c.turns[:len(turns)] = list(turns)
        self._ref = C.byref(self._c)

    axes = property(lambda self: self._c.axes)
    dim = property(lambda self: self._c.dim)
    turns = property(lambda self: list(self._c.turns[:self._c.dim // self._c.axes // 2]))


def fvar_rope_apply(ctx: Context, rope: Rope, pos, B: int, n: int, q=None, k=None, q_out=None, k_out=None, stream=None) -> None:
    """q: [B, n, heads, head_dim], k: [B, n, kv_heads, head_dim]; either may be None.  Rows may lie apart, as the parts of a fused
    projection's output do; without an output the rows are turned in place."""
    if B < 1 or n < 1:
        raise ValueError(f"B >= 1 and n >= 1 are wanted, got {B} and {n}")
    kind, kv_heads = _kind(ctx.dtype), ctx.heads if k is None else k.numel() // (B * n * ctx.head_dim)
    (qp, ldq), (kp, ldk) = _rows(q, kind, B, n, ctx.hidden), _rows(k, kind, B, n, kv_heads * ctx.head_dim)
    (qo, ldqo) = (qp, ldq) if q_out is None else _rows(q_out, kind, B, n, ctx.hidden)
    (ko, ldko) = (kp, ldk) if k_out is None else _rows(k_out, kind, B, n, kv_heads * ctx.head_dim)
    ctx.check(ctx.lib.fvar_rope_apply(ctx.handle, _stream(stream), rope._ref, _packed(pos, _kind("i32"), B, n, rope.axes), B, n, kv_heads,
                                      qp, ldq, kp, ldk, qo, ldqo, ko, ldko))


def fvar_kvb_append(ctx: Context, kv: KVB, k, v, B: int, rows: int, stream=None) -> None:
    kind, width = _kind(ctx.dtype), kv._c.kv_heads * ctx.head_dim
    (kp, ldk), (vp, ldv) = _rows(k, kind, B, rows, width), _rows(v, kind, B, rows, width)
    if (ldk or width) != (ldv or width):
        raise ValueError("k and v have different distances between rows")
    ctx.check(ctx.lib.fvar_kvb_append(ctx.handle, _stream(stream), kv._for(ctx, B), kp, vp, ldk, B, rows))


def fvar_kvb_read(ctx: Context, kv: KVB, B: int, first: int, rows: int, k=None, v=None, stream=None) -> None:
    kind, width = _kind(ctx.dtype), kv._c.kv_heads * ctx.head_dim
    kp, vp = _packed(k, kind, B, rows, width), _packed(v, kind, B, rows, width)
    ctx.check(ctx.lib.fvar_kvb_read(ctx.handle, _stream(stream), kv._for(ctx, B), B, first, rows, kp, vp))


def fvar_kvb_attention_workspace_bytes(ctx: Context, kv: KVB, B: int, n: int, weights: bool = False) -> int:
    return ctx.lib.fvar_kvb_attention_workspace_bytes(ctx.handle, kv._for(ctx, B), B, n, 1 if weights else 0)


def _row_weights(t, kv: KVB, B: int) -> Optional[int]:
    """Pointer of contiguous fp32 [B, kv_heads, capacity] (None passes NULL)."""
    return _packed(t, _kind("f32"), B, kv.kv_heads * kv.capacity, 1)


def fvar_kvb_attention(ctx: Context, q, kv: KVB, B: int, n: int, o, ws=None, weights=None, add: bool = False, stream=None) -> None:
    kind = _kind(ctx.dtype)
    qp, ld = _rows(q, kind, B, n, ctx.hidden)
    op = _packed(o, kind, B, n, ctx.hidden)
    ctx.check(ctx.lib.fvar_kvb_attention(ctx.handle, _stream(stream), qp, ld, kv._for(ctx, B), B, n, op, _row_weights(weights, kv, B),
                                         1 if add else 0, _ptr(ws), _nbytes(ws)))


def fvar_block_kvb_workspace_bytes(ctx: Context, kv: KVB, B: int, rows: int, weights: bool = False) -> int:
    return ctx.lib.fvar_block_kvb_workspace_bytes(ctx.handle, kv._for(ctx, B), B, rows, 1 if weights else 0)


def _turned(rope: Optional[Rope], pos, B: int, rows: int):
    if rope is None:
        if pos is not None:
            raise ValueError("positions without rope")
        return None, None
    return rope._ref, _packed(pos, _kind("i32"), B, rows, rope.axes)


def fvar_block_forward_dense_kvb(ctx: Context, w: dict, x, B: int, M: int, kv: KVB, y, ws, rope: Optional[Rope] = None, pos=None, weights=None,
                                 add: bool = False, stream=None) -> None:
    ws_, kind, (rp, pp) = _weights(w), _kind(ctx.dtype), _turned(rope, pos, B, M)
    xp, yp = _packed(x, kind, B, M, ctx.hidden), _packed(y, kind, B, M, ctx.hidden)
    ctx.check(ctx.lib.fvar_block_forward_dense_kvb(ctx.handle, _stream(stream), C.byref(ws_), xp, B, M, kv._for(ctx, B), rp, pp,
                                                   _row_weights(weights, kv, B), 1 if add else 0, yp, _ptr(ws), _nbytes(ws)))


def fvar_block_forward_pruned_kvb(ctx: Context, w: dict, x, B: int, M: int, idx_keep, k: int, kv: KVB, y_keep, ws, rope: Optional[Rope] = None,
                                  pos=None, weights=None, add: bool = False, stream=None) -> None:
    ws_, kind, (rp, pp) = _weights(w), _kind(ctx.dtype), _turned(rope, pos, B, k)
    xp, yp = _packed(x, kind, B, M, ctx.hidden), _packed(y_keep, kind, B, k, ctx.hidden)
    ctx.check(ctx.lib.fvar_block_forward_pruned_kvb(ctx.handle, _stream(stream), C.byref(ws_), xp, B, M,
                                                    _packed(idx_keep, _kind("i32"), B, k, 1), k, kv._for(ctx, B), rp, pp,
                                                    _row_weights(weights, kv, B), 1 if add else 0, yp, _ptr(ws), _nbytes(ws)))


def fvar_kvb_evict_workspace_bytes(ctx: Context, kv: KVB, B: int, keep: int) -> int:
    return ctx.lib.fvar_kvb_evict_workspace_bytes(ctx.handle, kv._for(ctx, B), B, keep)


def fvar_kvb_evict(ctx: Context, kv: KVB, weights, B: int, keep: int, recent: int, to: KVB, to_weights, to_lens=None, idx=None, ws=None,
                   stream=None) -> None:
    """to is kv itself, or shares no memory with it.  The lengths and the mask stay the caller's: afterwards to.lens is to_lens (or to.len `keep`, where every
    sample held as many rows that are not hidden), and to.mask None."""
    ctx.check(ctx.lib.fvar_kvb_evict(ctx.handle, _stream(stream), kv._for(ctx, B), _row_weights(weights, kv, B), B, keep, recent,
                                     to._for(ctx, B), _row_weights(to_weights, to, B), _packed(to_lens, _kind("i32"), B, 1, 1),
                                     _packed(idx, _kind("i32"), B, kv.kv_heads * keep, 1), _ptr(ws), _nbytes(ws)))


def fvar_profile_enable(ctx: Context, on: bool) -> None:
    ctx.check(ctx.lib.fvar_profile_enable(ctx.handle, 1 if on else 0))


def fvar_profile_read(ctx: Context) -> dict:
    """{label: (launches, total_ms)} since the last read."""
    buf = (_ProfileEntry * 64)()
    n = ctx.lib.fvar_profile_read(ctx.handle, buf, 64)
    return {buf[i].label.decode(): (int(buf[i].launches), float(buf[i].total_ms))
            for i in range(min(n, 64))}
