"""ctypes binding of the entry points behind the compressed rows (see ``include/ttf.h``): norm and
rotation of queries and keys, cache append, attention over a paged cache.  Argument marshalling only.

For inference: nothing is kept for a backward pass.  Outputs carry no gradient, also where an input requires one, and what is
written in place (``q_out``, ``k_out``, ``out``, ``lse``, the cache) changes without autograd's knowledge."""
from __future__ import annotations

import ctypes
import struct
from dataclasses import dataclass
from typing import Optional, Sequence

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


def _packer(structure):
    """Packs the fields of a ctypes structure, in order, into bytes of its layout (several times faster than filling it, which
    would also cut off numbers of more bits than a field has)."""
    codes = {_i32: "i", _i64: "q", _vp: "P", _f32: "f"}
    layout = "@" + "".join(codes[kind] for _, kind in structure._fields_)
    pad = ctypes.sizeof(structure) - struct.calcsize(layout)
    pack = struct.Struct(layout + (f"{pad}x" if pad else "")).pack

    def checked(*values):
        try:
            return pack(*values)
        except (struct.error, OverflowError) as error:
            raise ValueError(f"an argument is no number or does not fit its field: {error}") from None
    return checked


_pack_qk, _pack_cache, _pack_attention = _packer(_QKParams), _packer(_KVCache), _packer(_AttentionParams)

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


def _dtype_code(dtype: torch.dtype) -> int:
    code = _DTYPES.get(dtype)
    if code is None:
        raise TypeError(f"expected bfloat16 or float32, got {dtype}")
    return code


def _heads(name: str, x: torch.Tensor, rows: int, D: int, dtype: torch.dtype, gpu: int):
    """(address, heads, row stride, head stride) of a [rows, heads, D] operand."""
    shape, strides = x.shape, x.stride()
    if len(shape) != 3 or shape[0] != rows or shape[2] != D or x.dtype is not dtype or x.get_device() != gpu:
        raise ValueError(f"{name} must be [rows, heads, head_dim] with the rows, head_dim, dtype and device of the other operands")
    if strides[2] != 1 and D > 1:
        raise ValueError(f"{name} must have contiguous heads")
    return x.data_ptr(), shape[1], strides[0], strides[1]


def _vector(name: str, x: torch.Tensor, entries: int, dtype: torch.dtype, gpu: int) -> int:
    """Address of a contiguous vector."""
    if x.dtype is not dtype or x.dim() != 1 or x.shape[0] != entries or x.get_device() != gpu or (entries > 1 and x.stride(0) != 1):
        raise ValueError(f"{name} must be a contiguous [{entries}] tensor of {dtype} on the operands' device")
    return x.data_ptr()


def _empty(shape, dtype, device, stream) -> torch.Tensor:
    """Memory that the call's own stream may use at once, and after which torch may give it to that stream again."""
    if stream is None or device.type != "cuda":
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _call(function, gpu: int, stream, *args) -> None:
    if gpu < 0:
        raise ValueError("tensors must live on the GPU (the library has no CPU path)")
    if gpu == torch.cuda.current_device():
        _check(function(*args, _current_stream(gpu) if stream is None else stream.cuda_stream))
    else:
        with torch.cuda.device(gpu):
            _check(function(*args, _current_stream(gpu) if stream is None else stream.cuda_stream))


# address of the current stream, without making a torch.cuda.Stream for it
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda gpu: torch.cuda.current_stream(gpu).cuda_stream)


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
    strides (``transpose(1, 2)`` of a cache that keeps heads first is fine), ``page_table`` int32 [batch, width].

    What the tensors hold may change between calls.  ``page_table`` may be set to another tensor (a wider one, or
    one of another batch), which the next call uses; other ``k`` and ``v`` are another cache.  Their addresses and
    sizes are taken down here: none of them may be resized in place."""

    __slots__ = ("_k", "_v", "_page_table", "_struct", "_batch", "_heads", "_head_dim", "_gpu")

    def __init__(self, k: torch.Tensor, v: torch.Tensor, page_table: torch.Tensor):
        shape, strides, gpu = k.shape, k.stride(), k.get_device()
        if len(shape) != 4 or shape != v.shape or strides != v.stride() or k.dtype is not v.dtype or strides[3] != 1:
            raise ValueError("k and v must be [pages, page_size, kv_heads, head_dim] with contiguous heads, alike in every way")
        if gpu != v.get_device():
            raise ValueError("k, v and page_table must live on one device")
        self._k, self._v, self._gpu = k, v, gpu
        self._heads, self._head_dim = shape[2], shape[3]
        self.page_table = page_table

    @property
    def k(self) -> torch.Tensor:
        return self._k

    @property
    def v(self) -> torch.Tensor:
        return self._v

    @property
    def page_table(self) -> torch.Tensor:
        return self._page_table

    @page_table.setter
    def page_table(self, page_table: torch.Tensor) -> None:
        if page_table.dim() != 2 or page_table.dtype is not torch.int32 or (page_table.shape[1] > 1 and page_table.stride(1) != 1):
            raise ValueError("page_table must be int32 [batch, width] with contiguous rows")
        if page_table.get_device() != self._gpu:
            raise ValueError("k, v and page_table must live on one device")
        k, (batch, width) = self._k, page_table.shape
        strides = k.stride()
        self._struct = _pack_cache(k.data_ptr(), self._v.data_ptr(), page_table.data_ptr(), strides[0], strides[1], strides[2],
                                   page_table.stride(0) if batch > 1 else width, k.shape[0], k.shape[1], width)
        self._page_table, self._batch = page_table, batch


_NONE = (0, 0, 0, 0)


def _qk_params(q, k, v, q_out, k_out, pos, rope, q_weight, k_weight, eps, row_offsets, cached, batch, append):
    """(packed parameters, device index, rows)."""
    ref = k if k is not None else q
    if ref is None or ref.dim() != 3:
        raise ValueError("q and k must be [rows, heads, head_dim]")
    (rows, _, D), dtype, gpu = ref.shape, ref.dtype, ref.get_device()
    code = _dtype_code(ref.dtype)
    qs, qo, ks, ko, vs = _NONE, _NONE, _NONE, _NONE, _NONE
    if q is not None:
        qs, qo = _heads("q", q, rows, D, dtype, gpu), _heads("q_out", q_out, rows, D, dtype, gpu)
        if qs[1] != qo[1]:
            raise ValueError("q_out must have the shape of q")
    if k is not None:
        ks = _heads("k", k, rows, D, dtype, gpu)
        other = vs = _heads("v", v, rows, D, dtype, gpu) if append else vs
        if not append:
            other = ko = _heads("k_out", k_out, rows, D, dtype, gpu)
        if ks[1] != other[1]:
            raise ValueError("v and k_out must have the heads of k")
    rot = layout = axes = freq = axis = where = stride = 0
    factor = 1.0
    if rope is not None:
        pairs = rope.inv_freq.numel()
        freq = _vector("inv_freq", rope.inv_freq, pairs, torch.float64, gpu)
        layout = _LAYOUTS.get(rope.layout)
        if layout is None:
            raise ValueError(f"layout must be one of {tuple(_LAYOUTS)}")
        if pos is None or pos.dtype is not torch.int32 or pos.get_device() != gpu:
            raise ValueError("pos must be an int32 tensor on the operands' device")
        shape, strides = pos.shape, pos.stride()
        if not 1 <= len(shape) <= 2 or shape[-1] < rows or (shape[-1] > 1 and strides[-1] != 1):
            raise ValueError("pos must be [axes, rows] (or [rows]), contiguous along the rows")
        axes = shape[0] if len(shape) == 2 else 1
        stride = strides[0] if axes > 1 else rows
        rot, where, factor = 2 * pairs, pos.data_ptr(), rope.attention_factor
        if rope.axis is not None:
            axis = _vector("axis", rope.axis, pairs, torch.int32, gpu)
    packed = _pack_qk(
        code, D, qs[1], ks[1], rows, batch,
        0 if row_offsets is None else _vector("row_offsets", row_offsets, batch + 1, torch.int32, gpu),
        0 if cached is None else _vector("cached", cached, batch, torch.int32, gpu),
        qs[0], ks[0], vs[0], qs[2], qs[3], ks[2], ks[3], vs[2], vs[3], qo[0], ko[0], qo[2], qo[3], ko[2], ko[3],
        0 if q_weight is None else _vector("q_weight", q_weight, D, dtype, gpu),
        0 if k_weight is None else _vector("k_weight", k_weight, D, dtype, gpu),
        eps, rot, layout, axes, freq, axis, where, stride, factor)
    return packed, gpu, rows


def ttf_qk_norm_rope(q: Optional[torch.Tensor], k: Optional[torch.Tensor], pos: Optional[torch.Tensor] = None,
                     rope: Optional[TTFRope] = None, q_weight: Optional[torch.Tensor] = None,
                     k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
                     row_offsets: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                     k_out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """Norm (where a weight is given) and rotation (where ``rope`` is given) of every head of ``q`` [rows, heads, D]
    and ``k`` [rows, kv_heads, D], either of which may be None, by the positions ``pos`` int32 [axes, rows].

    ``row_offsets`` [batch + 1] (as ``ttf_compress`` writes it): only its rows are worked on, rows behind the
    last sequence stay as they were.  ``q_out`` / ``k_out`` may be the inputs themselves.  Returns (q_out, k_out).  No gradients."""
    if q is not None and q_out is None:
        q_out = _empty(q.shape, q.dtype, q.device, stream)
    if k is not None and k_out is None:
        k_out = _empty(k.shape, k.dtype, k.device, stream)
    batch = max(1, row_offsets.numel() - 1) if row_offsets is not None else 1
    packed, gpu, rows = _qk_params(q, k, None, q_out, k_out, pos, rope, q_weight, k_weight, eps, row_offsets, None, batch, False)
    if rows:
        _call(_library().ttf_qk_norm_rope, gpu, stream, packed)
    return q_out, k_out


def ttf_cache_append(cache: TTFKVCache, k: torch.Tensor, v: torch.Tensor, row_offsets: torch.Tensor, cached: torch.Tensor,
                     pos: Optional[torch.Tensor] = None, rope: Optional[TTFRope] = None,
                     k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, q: Optional[torch.Tensor] = None,
                     q_weight: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                     stream: Optional[torch.cuda.Stream] = None) -> Optional[torch.Tensor]:
    """Put normed and rotated keys and the values of packed rows into ``cache``: row i of sequence b becomes entry
    ``cached[b] + i``.  ``q`` is normed and rotated in the same launch.  Returns q_out (None without q).  No gradients."""
    if cache._k.dtype is not k.dtype or cache._gpu != k.get_device() or (cache._heads, cache._head_dim) != tuple(k.shape[1:]):
        raise ValueError("the cache must have the heads, head_dim, dtype and device of k")
    if q is not None and q_out is None:
        q_out = _empty(q.shape, q.dtype, q.device, stream)
    packed, gpu, rows = _qk_params(q, k, v, q_out, None, pos, rope, q_weight, k_weight, eps, row_offsets, cached, cache._batch, True)
    if rows:
        _call(_library().ttf_cache_append, gpu, stream, packed, cache._struct)
    return q_out


def ttf_attention_workspace_size(rows: int, batch: int, heads: int, kv_heads: int, head_dim: int,
                                 dtype: torch.dtype = torch.bfloat16, max_rows: Optional[int] = None) -> int:
    """Bytes of workspace that ``ttf_paged_attention`` needs for such a call, and for every one with the same heads, head_dim and
    dtype and no more rows, sequences and ``max_rows`` (default: all rows)."""
    packed = _pack_attention(_dtype_code(dtype), head_dim, heads, kv_heads, rows, batch, rows if max_rows is None else max_rows, 1, 0, 1.0,
                             *(0,) * 9)
    n = ctypes.c_size_t(0)
    _check(_library().ttf_attention_workspace_size(packed, ctypes.byref(n)))
    return int(n.value)


def ttf_paged_attention(q: torch.Tensor, cache: TTFKVCache, row_offsets: torch.Tensor, cached: torch.Tensor,
                        max_rows: Optional[int] = None, scale: Optional[float] = None, causal: bool = True, window: int = 0,
                        out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                        workspace: Optional[torch.Tensor] = None,
                        stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Attention of the packed rows ``q`` [rows, heads, D] over ``cache``, whose sequences hold ``cached`` entries and these
    rows' own (``ttf_cache_append`` first).  ``max_rows`` (most rows of one sequence, at least 1; default: all) picks the kernel
    and with it the room taken in ``workspace`` (uint8, of ttf_attention_workspace_size; taken from torch where not given);
    ``scale`` defaults to 1/sqrt(D); ``window`` > 0: a row looks back over that many entries, itself included; ``lse``
    float32 [rows, heads] is filled where given.  Rows outside ``row_offsets`` stay as they were.  No gradients."""
    if q.dim() != 3:
        raise ValueError("q must be [rows, heads, head_dim]")
    (rows, heads, D), dtype, gpu = q.shape, q.dtype, q.get_device()
    if cache._k.dtype is not dtype or cache._gpu != gpu or cache._head_dim != D:
        raise ValueError("the cache must have the head_dim, dtype and device of q")
    if out is None:
        out = _empty((rows, heads, D), dtype, q.device, stream)
    at, _, row, head = _heads("q", q, rows, D, dtype, gpu)
    to, out_heads, out_row, out_head = _heads("out", out, rows, D, dtype, gpu)
    if out_heads != heads:
        raise ValueError("out must have the shape of q")
    if lse is not None and (lse.dtype is not torch.float32 or tuple(lse.shape) != (rows, heads) or lse.get_device() != gpu
                            or not lse.is_contiguous()):
        raise ValueError("lse must be a contiguous float32 [rows, heads] tensor on the device of q")
    batch = cache._batch
    packed = _pack_attention(_dtype_code(q.dtype), D, heads, cache._heads, rows, batch, rows if max_rows is None else max_rows,
                             1 if causal else 0, window, D ** -0.5 if scale is None else scale,
                             _vector("row_offsets", row_offsets, batch + 1, torch.int32, gpu),
                             _vector("cached", cached, batch, torch.int32, gpu),
                             at, to, 0 if lse is None else lse.data_ptr(), row, head, out_row, out_head)
    if rows == 0:
        return out
    lib = _library()
    if workspace is None:
        n = ctypes.c_size_t(0)
        _check(lib.ttf_attention_workspace_size(packed, ctypes.byref(n)))
        workspace = _empty(n.value, torch.uint8, q.device, stream)
    elif workspace.get_device() != gpu or workspace.dtype is not torch.uint8 or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor on the device of q")
    base = workspace.data_ptr()
    skip = -base % 256
    _call(lib.ttf_paged_attention, gpu, stream, packed, cache._struct, base + skip, max(0, workspace.numel() - skip))
    return out
