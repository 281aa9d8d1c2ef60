"""ctypes binding of the entry points behind the compressed rows (see ``include/ttf.h``): norm and
rotation of queries and keys, cache append, attention over a paged cache.  Argument marshalling only."""
from __future__ import annotations

import ctypes
import math
from dataclasses import dataclass
from typing import Optional, Sequence, Tuple

import torch

from .binding import TTF_BF16, TTF_F32, _check, load_library

TTF_ROPE_HALF, TTF_ROPE_INTERLEAVED = 0, 1
_LAYOUTS = {"half": TTF_ROPE_HALF, "interleaved": TTF_ROPE_INTERLEAVED}
_SCALINGS = {"plain": 0, "linear": 1, "base": 2, "parts": 3, "turns": 4}
_DTYPES = {torch.bfloat16: TTF_BF16, torch.float32: TTF_F32}

_i32, _i64, _vp, _f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_float


class _QKParams(ctypes.Structure):
    _fields_ = ([(n, _i32) for n in ("dtype", "head_dim", "heads", "kv_heads", "rows", "batch")]
                + [(n, _vp) for n in ("row_offsets", "cached", "q", "k", "v")]
                + [(n, _i64) for n in ("q_row", "q_head", "k_row", "k_head", "v_row", "v_head")]
                + [(n, _vp) for n in ("q_out", "k_out")]
                + [(n, _i64) for n in ("qo_row", "qo_head", "ko_row", "ko_head")]
                + [("q_weight", _vp), ("k_weight", _vp), ("eps", _f32)]
                + [(n, _i32) for n in ("rotary_dim", "layout", "axes")]
                + [(n, _vp) for n in ("inv_freq", "axis", "pos")]
                + [("pos_stride", _i64), ("attention_factor", _f32)])


class _KVCache(ctypes.Structure):
    _fields_ = ([(n, _vp) for n in ("k", "v", "page_table")]
                + [(n, _i64) for n in ("page_stride", "slot_stride", "head_stride", "table_stride")]
                + [(n, _i32) for n in ("pages", "page_size", "table_width")])


class _AttentionParams(ctypes.Structure):
    _fields_ = ([(n, _i32) for n in ("dtype", "head_dim", "heads", "kv_heads", "rows", "batch", "max_rows", "causal",
                                     "window")]
                + [("scale", _f32)] + [(n, _vp) for n in ("row_offsets", "cached", "q", "out", "lse")]
                + [(n, _i64) for n in ("q_row", "q_head", "o_row", "o_head")])


_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = load_library()
        lib.ttf_rope_table.restype = ctypes.c_int
        lib.ttf_rope_table.argtypes = [_i32, ctypes.c_double, _i32] + [ctypes.c_double] * 4 + [_i32, _vp, _i32, _vp, _vp, _vp]
        for name, args in (("ttf_qk_norm_rope", [_vp, _vp]), ("ttf_cache_append", [_vp, _vp, _vp]),
                           ("ttf_attention_workspace_size", [_vp, _vp]),
                           ("ttf_paged_attention", [_vp, _vp, _vp, ctypes.c_size_t, _vp])):
            f = getattr(lib, name)
            f.restype, f.argtypes = ctypes.c_int, args
        _lib = lib
    return _lib


def _dtype_of(x: torch.Tensor) -> int:
    code = _DTYPES.get(x.dtype)
    if code is None:
        raise TypeError(f"expected bfloat16 or float32, got {x.dtype}")
    return code


def _heads(name: str, x: torch.Tensor, like: torch.Tensor) -> None:
    if x.dim() != 3 or x.stride(2) != 1 and x.shape[2] > 1:
        raise ValueError(f"{name} must be [rows, heads, head_dim] with contiguous heads")
    if x.dtype != like.dtype or x.device != like.device or x.shape[2] != like.shape[2] or x.shape[0] != like.shape[0]:
        raise ValueError(f"{name} must have the rows, head_dim, dtype and device of the other operands")


def _ints(name: str, x: torch.Tensor, entries: int, device) -> int:
    if x.dtype != torch.int32 or x.dim() != 1 or x.numel() != entries or x.device != device or (entries > 1 and x.stride(0) != 1):
        raise ValueError(f"{name} must be a contiguous int32 [{entries}] tensor on {device}")
    return x.data_ptr()


def _empty(shape, dtype, device, stream) -> torch.Tensor:
    """Memory that the call's own stream may use at once, and after which torch may give it to that stream again."""
    if stream is None or device.type != "cuda":
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _call(function, device: torch.device, stream, *args) -> None:
    if not device.type == "cuda":
        raise ValueError("tensors must live on the GPU (the library has no CPU path)")
    if device.index == torch.cuda.current_device():
        s = torch.cuda.current_stream(device) if stream is None else stream
        _check(function(*args, s.cuda_stream))
    else:
        with torch.cuda.device(device):
            s = torch.cuda.current_stream(device) if stream is None else stream
            _check(function(*args, s.cuda_stream))


@dataclass
class TTFRope:
    """The rotation of a head: frequencies of its pairs, the position plane each pair goes by, the layout
    of the pairs ("half": (j, j + R/2), "interleaved": (2j, 2j + 1)) and the factor on sine and cosine."""
    inv_freq: torch.Tensor                 # [R/2] float64
    axis: Optional[torch.Tensor] = None    # [R/2] int32; None: plane 0
    layout: str = "half"
    attention_factor: float = 1.0


def ttf_rope_table(rotary_dim: int, base: float = 10000.0, scaling: str = "plain", factor: float = 1.0,
                   original_length: float = 0.0, fast: float = 32.0, slow: float = 1.0,
                   sections: Optional[Sequence[int]] = None, take_turns: bool = False, layout: str = "half",
                   device="cuda") -> TTFRope:
    """Frequencies of ``rotary_dim / 2`` pairs, scaled for long contexts, and the planes they go by
    (``sections``: pairs of each plane, in blocks or taking turns).  Computed on the host, kept on ``device``."""
    if scaling not in _SCALINGS:
        raise ValueError(f"scaling must be one of {tuple(_SCALINGS)}")
    if layout not in _LAYOUTS:
        raise ValueError(f"layout must be one of {tuple(_LAYOUTS)}")
    half = max(1, int(rotary_dim) // 2)
    freq, plane, attention = (ctypes.c_double * half)(), (_i32 * half)(), _f32(1.0)
    parts = (_i32 * len(sections))(*(int(n) for n in sections)) if sections is not None else None
    _check(_library().ttf_rope_table(int(rotary_dim), float(base), _SCALINGS[scaling], float(factor), float(original_length),
                                     float(fast), float(slow), 1 if parts is None else len(parts), parts, int(take_turns),
                                     freq, plane, ctypes.byref(attention)))
    return TTFRope(torch.tensor(list(freq), dtype=torch.float64, device=device),
                   torch.tensor(list(plane), dtype=torch.int32, device=device) if parts is not None else None,
                   layout, float(attention.value))


class TTFKVCache:
    """A paged cache: ``k`` and ``v`` [pages, page_size, kv_heads, head_dim] with contiguous heads and the same
    strides (``transpose(1, 2)`` of a cache that keeps heads first is fine), ``page_table`` int32 [batch, width]."""

    __slots__ = ("k", "v", "page_table", "_struct")

    def __init__(self, k: torch.Tensor, v: torch.Tensor, page_table: torch.Tensor):
        if k.dim() != 4 or k.shape != v.shape or k.stride() != v.stride() or k.dtype != v.dtype or k.stride(3) != 1:
            raise ValueError("k and v must be [pages, page_size, kv_heads, head_dim] with contiguous heads, alike in every way")
        if page_table.dim() != 2 or page_table.dtype != torch.int32 or (page_table.shape[1] > 1 and page_table.stride(1) != 1):
            raise ValueError("page_table must be int32 [batch, width] with contiguous rows")
        if not k.device == v.device == page_table.device:
            raise ValueError("k, v and page_table must live on one device")
        self.k, self.v, self.page_table = k, v, page_table
        pages, size = k.shape[:2]
        sp, ss, sh, _ = k.stride()
        width = page_table.shape[1]
        stride = page_table.stride(0) if page_table.shape[0] > 1 else width
        self._struct = _KVCache(k.data_ptr(), v.data_ptr(), page_table.data_ptr(), sp, ss, sh, stride, pages, size, width)


def _qk_params(q, k, v, q_out, k_out, pos, rope, q_weight, k_weight, eps, row_offsets, cached, batch) -> Tuple[_QKParams, torch.device]:
    ref = k if k is not None else q
    if ref is None or ref.dim() != 3:
        raise ValueError("q and k must be [rows, heads, head_dim]")
    rows, _, D = ref.shape
    device = ref.device
    p = _QKParams(_dtype_of(ref), D, 0, 0, rows, batch, None, None)
    if row_offsets is not None:
        p.row_offsets = _ints("row_offsets", row_offsets, batch + 1, device)
    if cached is not None:
        p.cached = _ints("cached", cached, batch, device)
    if q is not None:
        _heads("q", q, ref)
        _heads("q_out", q_out, ref)
        p.heads, p.q, p.q_out = q.shape[1], q.data_ptr(), q_out.data_ptr()
        p.q_row, p.q_head, _ = q.stride()
        p.qo_row, p.qo_head, _ = q_out.stride()
        if q_out.shape[1] != q.shape[1]:
            raise ValueError("q_out must have the shape of q")
    if k is not None:
        _heads("k", k, ref)
        p.kv_heads, p.k = k.shape[1], k.data_ptr()
        p.k_row, p.k_head, _ = k.stride()
        if k_out is not None:
            _heads("k_out", k_out, ref)
            if k_out.shape[1] != k.shape[1]:
                raise ValueError("k_out must have the shape of k")
            p.k_out = k_out.data_ptr()
            p.ko_row, p.ko_head, _ = k_out.stride()
        if v is not None:
            _heads("v", v, ref)
            if v.shape[1] != k.shape[1]:
                raise ValueError("v must have the heads of k")
            p.v = v.data_ptr()
            p.v_row, p.v_head, _ = v.stride()
    for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
        if w is not None:
            if w.dtype != ref.dtype or w.dim() != 1 or w.numel() != D or w.device != device or (D > 1 and w.stride(0) != 1):
                raise ValueError(f"{name} must be a contiguous [head_dim] tensor of the operands' dtype")
            setattr(p, name, w.data_ptr())
    p.eps = eps
    if rope is not None:
        f, axis = rope.inv_freq, rope.axis
        if f.dtype != torch.float64 or f.dim() != 1 or f.device != device or (f.numel() > 1 and f.stride(0) != 1):
            raise ValueError("inv_freq must be a contiguous float64 [rotary_dim / 2] tensor on the operands' device")
        if pos is None or pos.dtype != torch.int32 or pos.device != device:
            raise ValueError("pos must be an int32 tensor on the operands' device")
        if pos.dim() == 1:
            pos = pos[None]
        if pos.dim() != 2 or pos.shape[1] < rows or (pos.shape[1] > 1 and pos.stride(1) != 1):
            raise ValueError("pos must be [axes, rows] (or [rows]), contiguous along the rows")
        if rope.layout not in _LAYOUTS:
            raise ValueError(f"layout must be one of {tuple(_LAYOUTS)}")
        p.rotary_dim, p.layout, p.axes = 2 * f.numel(), _LAYOUTS[rope.layout], pos.shape[0]
        p.inv_freq, p.pos = f.data_ptr(), pos.data_ptr()
        p.pos_stride = pos.stride(0) if pos.shape[0] > 1 else rows
        p.attention_factor = rope.attention_factor
        if axis is not None:
            p.axis = _ints("axis", axis, f.numel(), device)
    return p, device


def ttf_qk_norm_rope(q: Optional[torch.Tensor], k: Optional[torch.Tensor], pos: Optional[torch.Tensor] = None,
                     rope: Optional[TTFRope] = None, q_weight: Optional[torch.Tensor] = None,
                     k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
                     row_offsets: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                     k_out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """Norm (where a weight is given) and rotation (where ``rope`` is given) of every head of ``q`` [rows, heads, D]
    and ``k`` [rows, kv_heads, D], either of which may be None, by the positions ``pos`` int32 [axes, rows].

    ``row_offsets`` [batch + 1] (as ``ttf_compress`` writes it): only its rows are worked on, rows behind the
    last sequence stay as they were.  ``q_out`` / ``k_out`` may be the inputs themselves.  Returns (q_out, k_out)."""
    if q is not None and q_out is None:
        q_out = _empty(q.shape, q.dtype, q.device, stream)
    if k is not None and k_out is None:
        k_out = _empty(k.shape, k.dtype, k.device, stream)
    batch = max(1, row_offsets.numel() - 1) if row_offsets is not None else 1
    p, device = _qk_params(q, k, None, q_out, k_out, pos, rope, q_weight, k_weight, eps, row_offsets, None, batch)
    if p.rows:
        _call(_library().ttf_qk_norm_rope, device, stream, ctypes.byref(p))
    return q_out, k_out


def ttf_cache_append(cache: TTFKVCache, k: torch.Tensor, v: torch.Tensor, row_offsets: torch.Tensor, cached: torch.Tensor,
                     pos: Optional[torch.Tensor] = None, rope: Optional[TTFRope] = None,
                     k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, q: Optional[torch.Tensor] = None,
                     q_weight: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                     stream: Optional[torch.cuda.Stream] = None) -> Optional[torch.Tensor]:
    """Put normed and rotated keys and the values of packed rows into ``cache``: row i of sequence b becomes entry
    ``cached[b] + i``.  ``q`` is normed and rotated in the same launch.  Returns q_out (None without q)."""
    batch = cache.page_table.shape[0]
    if cache.k.dtype != k.dtype or cache.k.device != k.device or tuple(cache.k.shape[2:]) != tuple(k.shape[1:]):
        raise ValueError("the cache must have the heads, head_dim, dtype and device of k")
    if q is not None and q_out is None:
        q_out = _empty(q.shape, q.dtype, q.device, stream)
    p, device = _qk_params(q, k, v, q_out, None, pos, rope, q_weight, k_weight, eps, row_offsets, cached, batch)
    if p.rows:
        _call(_library().ttf_cache_append, device, stream, ctypes.byref(p), ctypes.byref(cache._struct))
    return q_out


def _attention_params(q, out, lse, cache, row_offsets, cached, max_rows, scale, causal, window) -> _AttentionParams:
    rows, heads, D = q.shape
    sq, so = q.stride(), out.stride()
    return _AttentionParams(_dtype_of(q), D, heads, cache.k.shape[2], rows, cache.page_table.shape[0],
                            rows if max_rows is None else max_rows, 1 if causal else 0, window,
                            D ** -0.5 if scale is None else scale, row_offsets, cached, q.data_ptr(), out.data_ptr(), lse,
                            sq[0], sq[1], so[0], so[1])


def ttf_attention_workspace_size(rows: int, batch: int, heads: int, kv_heads: int, head_dim: int,
                                 dtype: torch.dtype = torch.bfloat16, max_rows: Optional[int] = None) -> int:
    p = _AttentionParams(_DTYPES[dtype], head_dim, heads, kv_heads, rows, batch, rows if max_rows is None else max_rows, 1, 0, 1.0)
    n = ctypes.c_size_t(0)
    _check(_library().ttf_attention_workspace_size(ctypes.byref(p), ctypes.byref(n)))
    return int(n.value)


def ttf_paged_attention(q: torch.Tensor, cache: TTFKVCache, row_offsets: torch.Tensor, cached: torch.Tensor,
                        max_rows: Optional[int] = None, scale: Optional[float] = None, causal: bool = True, window: int = 0,
                        out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                        workspace: Optional[torch.Tensor] = None,
                        stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Attention of the packed rows ``q`` [rows, heads, D] over ``cache``, whose sequences hold ``cached`` entries and these
    rows' own (``ttf_cache_append`` first).  ``max_rows`` (most rows of one sequence; default: all) picks the kernel;
    ``scale`` defaults to 1/sqrt(D); ``window`` > 0: a row looks back over that many entries, itself included; ``lse``
    float32 [rows, heads] is filled where given.  Rows outside ``row_offsets`` stay as they were."""
    if q.dim() != 3 or q.stride(2) != 1 and q.shape[2] > 1:
        raise ValueError("q must be [rows, heads, head_dim] with contiguous heads")
    device = q.device
    if cache.k.dtype != q.dtype or cache.k.device != device or cache.k.shape[3] != q.shape[2]:
        raise ValueError("the cache must have the head_dim, dtype and device of q")
    batch = cache.page_table.shape[0]
    offsets, have = _ints("row_offsets", row_offsets, batch + 1, device), _ints("cached", cached, batch, device)
    if out is None:
        out = _empty(q.shape, q.dtype, device, stream)
    elif out.shape != q.shape or out.dtype != q.dtype or out.device != device or out.stride(2) != 1 and out.shape[2] > 1:
        raise ValueError("out must be like q, with contiguous heads")
    if lse is not None and (lse.dtype != torch.float32 or tuple(lse.shape) != tuple(q.shape[:2]) or lse.device != device
                            or not lse.is_contiguous()):
        raise ValueError("lse must be a contiguous float32 [rows, heads] tensor")
    if q.shape[0] == 0:
        return out
    p = _attention_params(q, out, None if lse is None else lse.data_ptr(), cache, offsets, have, max_rows, scale, causal, int(window))
    lib, ref = _library(), ctypes.byref(p)
    if workspace is None:
        n = ctypes.c_size_t(0)
        _check(lib.ttf_attention_workspace_size(ref, ctypes.byref(n)))
        workspace = _empty(n.value, torch.uint8, device, stream)
    elif workspace.device != device or workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor on the device of q")
    base = workspace.data_ptr()
    skip = -base % 256
    _call(lib.ttf_paged_attention, device, stream, ref, ctypes.byref(cache._struct), base + skip, max(0, workspace.numel() - skip))
    return out
