"""Tokens of a transformer behind a stage, for callers that hold torch tensors: positions of the patches of
packed crops, norm and rotation of query and key heads, attention to another set's states.

Argument checks and marshalling only; the work is done by octo_patch_positions, octo_norm_rotate and
octo_cross_attention of the C ABI (include/octo.h has the rules).  Calls enqueue on the current stream of the
tensors' device, or on `stream`; nothing synchronises, and a call may be captured into a CUDA graph.  What a call
allocates belongs to the stream it runs on; inputs have to be ready there, and may be dropped as soon as the call
returns.  There is no backward pass: results carry no gradient history."""
from __future__ import annotations

import ctypes
import struct
from typing import Optional, Tuple

from . import binding as B

# Marshalling is what a small call costs, so arguments are packed in one go (the layouts of octo_rotate_t and
# octo_attend_t) and what can be looked up once is.
_ROTATE = struct.Struct("@10iq" + "Pqq" * 4 + "6Pqff")
_ATTEND = struct.Struct("@6i2q" + "Pqq" * 4 + "2P6qPffP")
assert _ROTATE.size == ctypes.sizeof(B.Rotate) and _ATTEND.size == ctypes.sizeof(B.Attend)


class _Torch:
    """torch and what is asked of it in every call; filled by the first."""
    module = None
    types: dict = {}
    streams: dict = {}


def _torch():
    if _Torch.module is None:
        import torch
        _Torch.types = {torch.float16: B.OCTO_F16, torch.bfloat16: B.OCTO_BF16, torch.float32: B.OCTO_F32}
        _Torch.module = torch
    return _Torch.module


def _refuse(where: str, why: str):
    raise B.OctoError(B.OCTO_E_INVALID_ARG, f"{where} ({why})")


def _stream_of(device, stream) -> int:
    if stream is not None:
        return int(stream.cuda_stream)
    get = _Torch.streams.get(device.index)
    if get is None:
        get = _Torch.streams[device.index] = B._stream_getter(_torch(), device)
    return get()


def _on_device(where, device, *tensors) -> None:
    """Every tensor given lies on `device`: a pointer of another one would be read there."""
    index = device.index
    for t in tensors:
        if t is not None and t.get_device() != index:
            _refuse(where, f"a tensor is on {t.device}, not on {device}")


def _int32_vector(where, name, t, count) -> None:
    if t is not None and (t.dtype is not _Torch.module.int32 or t.dim() != 1 or t.shape[0] < count or t.stride(0) != 1):
        _refuse(where, f"{name} is not a contiguous int32 vector of at least {count}")


def patch_positions(items, slot: Tuple[int, int], patch: int, *, keep_aspect: bool = False, times=None, n_items=None,
                    positions=None, visible=None, stream=None):
    """Where the patches of packed crops lie (octo_patch_positions).

    items: item table on the GPU, int32 [n, 8] or uint8 [n, 32]; slot: (width, height) of a crop; times: float32
    [frames] or None; n_items: int32 {packed, ...} on the GPU or None (all of them).  Returns (positions float32
    [n, patches, 3], visible uint8 [n, patches]); rows of items beyond n_items are not written."""
    t, where = _torch(), "patch_positions"
    if not (items.is_cuda and items.dim() == 2 and items.is_contiguous()
            and (items.dtype, items.shape[1]) in ((t.int32, 8), (t.uint8, 32))):
        _refuse(where, "items is not a contiguous CUDA tensor of item records")
    n, (w, h) = items.shape[0], slot
    if not (patch > 0 and w > 0 and h > 0 and w % patch == 0 and h % patch == 0):
        _refuse(where, "the patch does not divide the slot")
    dev, patches = items.device, (w // patch) * (h // patch)
    if positions is None:
        positions = B._empty(t, (n, patches, 3), t.float32, dev, stream)
    if visible is None:
        visible = B._empty(t, (n, patches), t.uint8, dev, stream)
    if positions.dtype is not t.float32 or not positions.is_contiguous() or positions.numel() != n * patches * 3:
        _refuse(where, "positions has another shape")
    if visible.dtype is not t.uint8 or not visible.is_contiguous() or visible.numel() != n * patches:
        _refuse(where, "visible has another shape")
    if times is not None and (times.dtype is not t.float32 or times.dim() != 1 or not times.is_contiguous()):
        _refuse(where, "times is not a contiguous float32 vector")
    _int32_vector(where, "n_items", n_items, 1)
    _on_device(where, dev, times, n_items, positions, visible)
    # without times every frame number is one that exists
    frames = (1 << 31) - 1 if times is None else times.shape[0]
    rc = B.load_library().octo_patch_positions(
        dev.index, items.data_ptr(), n, None if n_items is None else n_items.data_ptr(), w, h, patch,
        1 if keep_aspect else 0, None if times is None else times.data_ptr(), frames, positions.data_ptr(),
        visible.data_ptr(), _stream_of(dev, stream))
    if rc != B.OCTO_OK:
        raise B.OctoError(rc, "octo_patch_positions")
    B._in_use(stream, items, times, n_items, positions, visible)
    return positions, visible


def norm_rotate(q, k, positions, freqs, axes, *, q_weight=None, k_weight=None, eps: float = 1e-6,
                interleaved: bool = False, n_items=None, item_rows: int = 1, out=None, stream=None):
    """Norm of every query and key head and its rotation by the token's position (octo_norm_rotate).

    q [rows, heads, dim], k [rows, kv_heads, dim] or None, of one type (float16, bfloat16, float32); the elements
    of a head lie side by side, rows and heads may have any stride.  positions: float32 or int32 [rows, axes];
    freqs float32 [pairs], axes int32 [pairs]: pair i turns by positions[:, axes[i]] * freqs[i].  q_weight,
    k_weight: [dim] of q's type, or None for no norm.  n_items (int32 on the GPU): rows from n_items * item_rows
    on are left as they were.  out: (q_out, k_out), which may be (q, k).  Returns (q_out, k_out)."""
    t, where = _torch(), "norm_rotate"
    dtype, dev = q.dtype, q.device
    code = _Torch.types.get(dtype)
    if code is None or not q.is_cuda or q.dim() != 3:
        _refuse(where, "q is not a CUDA tensor [rows, heads, dim]")
    rows, heads, dim = q.shape
    kv = 0
    if k is not None:
        if k.dim() != 3 or k.dtype is not dtype or k.shape[0] != rows or k.shape[2] != dim:
            _refuse(where, "k does not fit q")
        kv = k.shape[1]
    if out is None:
        out = (B._empty(t, (rows, heads, dim), dtype, dev, stream),
               None if k is None else B._empty(t, (rows, kv, dim), dtype, dev, stream))
    q_out, k_out = out
    views = []
    for x, y in ((q, q_out), (k, k_out)):
        if x is None:
            views += ((0, 0, 0), (0, 0, 0))
            continue
        if y is None or y.shape != x.shape or y.dtype is not dtype:
            _refuse(where, "an output has another shape than its input")
        (r0, h0, e0), (r1, h1, e1) = x.stride(), y.stride()
        if e0 != 1 or e1 != 1:
            _refuse(where, "the elements of a head are apart")
        views += ((x.data_ptr(), r0, h0), (y.data_ptr(), r1, h1))
    for w in (q_weight, k_weight):
        if w is not None and (w.dtype is not dtype or w.dim() != 1 or w.shape[0] != dim or w.stride(0) != 1):
            _refuse(where, "a weight is not a contiguous vector [dim] of q's type")
    if freqs.dim() != 1 or freqs.dtype is not t.float32 or not freqs.is_contiguous():
        _refuse(where, "freqs is not a float32 vector")
    pairs = freqs.shape[0]
    _int32_vector(where, "axes", axes, pairs)
    _int32_vector(where, "n_items", n_items, 1)
    whole = positions.dtype is t.int32
    if not (whole or positions.dtype is t.float32) or positions.dim() != 2 or positions.shape[0] != rows or not positions.is_contiguous():
        _refuse(where, "positions is not a contiguous float32 or int32 [rows, axes]")
    _on_device(where, dev, k, positions, freqs, axes, q_weight, k_weight, n_items, q_out, k_out)
    try:
        args = _ROTATE.pack(dev.index, code, heads, kv, dim, pairs, 1 if interleaved else 0, positions.shape[1], 1 if whole else 0,
                            0, rows, *views[0], *views[2], *views[1], *views[3],
                            0 if q_weight is None else q_weight.data_ptr(), 0 if k_weight is None else k_weight.data_ptr(),
                            positions.data_ptr(), freqs.data_ptr(), axes.data_ptr(), 0 if n_items is None else n_items.data_ptr(),
                            item_rows, eps, 0.0)
    except (struct.error, OverflowError) as e:
        _refuse(where, str(e))
    rc = B.load_library().octo_norm_rotate(args, _stream_of(dev, stream))
    if rc != B.OCTO_OK:
        raise B.OctoError(rc, "octo_norm_rotate")
    B._in_use(stream, q, k, positions, freqs, axes, q_weight, k_weight, n_items, q_out, k_out)
    return q_out, k_out


def cross_attention(q, k, v, segments: int, *, q_offsets=None, k_offsets=None, q_rows: int = 1, k_rows: int = 1,
                    q_first: int = 0, k_first: int = 0, max_q: Optional[int] = None, max_k: Optional[int] = None,
                    key_mask=None, scale: Optional[float] = None, out=None, status=None, stream=None):
    """Attention of q's tokens to the states k, v, segment by segment (octo_cross_attention).

    q [q_total, heads, dim], k and v [k_total, kv_heads, dim], float16 or bfloat16, dim a multiple of 8 up to 128.
    Segment s has query rows [(q_offsets[s] - q_first) * q_rows, (q_offsets[s + 1] - q_first) * q_rows) and key
    rows likewise; offsets are int32 [segments + 1] on the GPU (the ones octo_crop_batch wrote), without them
    segment s starts at row s * q_rows (s * k_rows).  max_q, max_k: the most rows a segment can have, where that
    is known (it lets the call split its work well); key_mask: uint8 or bool [k_total], 0 hides a key; scale:
    dim ** -0.5 unless given; status: uint32 or int32 [1] that collects OCTO_STATUS bits.  Rows of no segment are
    not written.  Returns out [q_total, heads, dim]."""
    t, where = _torch(), "cross_attention"
    dtype, dev = q.dtype, q.device
    if not q.is_cuda or q.dim() != 3 or dtype not in (t.float16, t.bfloat16):
        _refuse(where, "q is not a float16 or bfloat16 CUDA tensor [rows, heads, dim]")
    q_total, heads, dim = q.shape
    if k.dim() != 3 or k.shape != v.shape or k.shape[2] != dim or k.dtype is not dtype or v.dtype is not dtype:
        _refuse(where, "k and v do not fit q")
    k_total, kv, _ = k.shape
    if kv == 0 or heads % kv:
        _refuse(where, "kv_heads does not divide heads")
    if dim == 0:
        _refuse(where, "a head has no elements")
    if out is None:
        out = B._empty(t, (q_total, heads, dim), dtype, dev, stream)
    elif out.shape != q.shape or out.dtype is not dtype:
        _refuse(where, "out has another shape")
    views = []
    for x in (q, k, v, out):
        r, h, e = x.stride()
        if e != 1:
            _refuse(where, "the elements of a head are apart")
        # (the strides of a dimension of one or of none mean nothing)
        views += (x.data_ptr(), r if x.shape[0] > 1 else 0, h if x.shape[1] > 1 else 0)
    _int32_vector(where, "q_offsets", q_offsets, segments + 1)
    _int32_vector(where, "k_offsets", k_offsets, segments + 1)
    if key_mask is not None and (key_mask.dtype not in (t.uint8, t.bool) or key_mask.dim() != 1 or key_mask.shape[0] != k_total
                                 or not key_mask.is_contiguous()):
        _refuse(where, "key_mask is not a contiguous uint8 or bool [k_total]")
    if status is not None and (status.element_size() != 4 or status.numel() < 1):
        _refuse(where, "status is not a 32-bit word")
    _on_device(where, dev, k, v, out, q_offsets, k_offsets, key_mask, status)
    try:
        args = _ATTEND.pack(dev.index, _Torch.types[dtype], segments, heads, kv, dim, q_total, k_total, *views,
                            0 if q_offsets is None else q_offsets.data_ptr(), 0 if k_offsets is None else k_offsets.data_ptr(),
                            q_rows, k_rows, q_first, k_first, max_q or 0, max_k or 0,
                            0 if key_mask is None else key_mask.data_ptr(), dim ** -0.5 if scale is None else scale, 0.0,
                            0 if status is None else status.data_ptr())
    except (struct.error, OverflowError) as e:
        _refuse(where, str(e))
    lib = B.load_library()
    need = ctypes.c_int64()
    rc = lib.octo_attend_workspace(args, ctypes.byref(need))
    if rc != B.OCTO_OK:
        raise B.OctoError(rc, "octo_attend_workspace")
    workspace = B._empty(t, (need.value,), t.uint8, dev, stream) if need.value else None
    rc = lib.octo_cross_attention(args, None if workspace is None else workspace.data_ptr(), need.value, _stream_of(dev, stream))
    if rc != B.OCTO_OK:
        raise B.OctoError(rc, "octo_cross_attention")
    B._in_use(stream, q, k, v, q_offsets, k_offsets, key_mask, out, status)
    return out
