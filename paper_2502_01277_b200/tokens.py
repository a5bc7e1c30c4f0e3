"""Tokens of a transformer behind a stage, for callers that hold torch tensors: positions of the patches of
packed crops, norm and rotation of query and key heads, attention to another set's states.

Argument checks and marshalling only; the work is done by octo_patch_positions, octo_norm_rotate and
octo_cross_attention of the C ABI (include/octo.h has the rules).  Calls enqueue on the current stream of the
tensors' device, or on `stream`; nothing synchronises, and a call may be captured into a CUDA graph."""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

from . import binding as B

_DTYPES = {"torch.float16": B.OCTO_F16, "torch.bfloat16": B.OCTO_BF16, "torch.float32": B.OCTO_F32}
_streams = {}


def _refuse(where: str, why: str):
    raise B.OctoError(B.OCTO_E_INVALID_ARG, f"{where} ({why})")


def _need(ok: bool, where: str, why: str) -> None:
    if not ok:
        _refuse(where, why)


def _stream_of(torch, device, stream) -> int:
    if stream is not None:
        return int(stream.cuda_stream)
    get = _streams.get(device.index)
    if get is None:
        get = _streams[device.index] = B._stream_getter(torch, device)
    return get()


def _on_device(where, device, **tensors) -> None:
    """Every tensor given lies on `device`: a pointer of another one would be read there."""
    for name, t in tensors.items():
        if t is not None and t.device != device:
            _refuse(where, f"{name} is on {t.device}, not on {device}")


def _heads(t) -> B.Heads:
    h = B.Heads()
    h.d_data, h.row_stride, h.head_stride = t.data_ptr(), t.stride(0), t.stride(1)
    return h


def _int32_vector(where, name, t, count) -> None:
    if t is not None:
        _need(str(t.dtype) == "torch.int32" and t.dim() == 1 and t.numel() >= count and t.is_contiguous(), where,
              f"{name} is not a contiguous int32 vector of at least {count}")


def patch_positions(items, slot: Tuple[int, int], patch: int, *, keep_aspect: bool = False, times=None, n_items=None,
                    positions=None, visible=None, stream=None):
    """Where the patches of packed crops lie (octo_patch_positions).

    items: item table on the GPU, int32 [n, 8] or uint8 [n, 32]; slot: (width, height) of a crop; times: float32
    [frames] or None; n_items: int32 {packed, ...} on the GPU or None (all of them).  Returns (positions float32
    [n, patches, 3], visible uint8 [n, patches]); rows of items beyond n_items are not written."""
    import torch
    where = "patch_positions"
    _need(items.is_cuda and items.dim() == 2 and items.is_contiguous()
          and (items.dtype, items.shape[1]) in ((torch.int32, 8), (torch.uint8, 32)), where,
          "items is not a contiguous CUDA tensor of item records")
    n, (w, h) = items.shape[0], slot
    _need(patch > 0 and w > 0 and h > 0 and w % patch == 0 and h % patch == 0, where, "the patch does not divide the slot")
    dev, patches = items.device, (w // patch) * (h // patch)
    if positions is None:
        positions = torch.empty((n, patches, 3), dtype=torch.float32, device=dev)
    if visible is None:
        visible = torch.empty((n, patches), dtype=torch.uint8, device=dev)
    _need(positions.dtype == torch.float32 and positions.is_contiguous() and positions.numel() == n * patches * 3, where,
          "positions has another shape")
    _need(visible.dtype == torch.uint8 and visible.is_contiguous() and visible.numel() == n * patches, where,
          "visible has another shape")
    _need(times is None or (times.dtype == torch.float32 and times.dim() == 1 and times.is_contiguous()), where,
          "times is not a contiguous float32 vector")
    _int32_vector(where, "n_items", n_items, 1)
    _on_device(where, dev, times=times, n_items=n_items, positions=positions, visible=visible)
    # without times every frame number is one that exists
    frames = (1 << 31) - 1 if times is None else times.numel()
    rc = B.load_library().octo_patch_positions(
        dev.index, items.data_ptr(), n, None if n_items is None else n_items.data_ptr(), w, h, patch,
        1 if keep_aspect else 0, None if times is None else times.data_ptr(), frames, positions.data_ptr(),
        visible.data_ptr(), _stream_of(torch, dev, stream))
    if rc != B.OCTO_OK:
        raise B.OctoError(rc, "octo_patch_positions")
    return positions, visible


def norm_rotate(q, k, positions, freqs, axes, *, q_weight=None, k_weight=None, eps: float = 1e-6,
                interleaved: bool = False, n_items=None, item_rows: int = 1, out=None, stream=None):
    """Norm of every query and key head and its rotation by the token's position (octo_norm_rotate).

    q [rows, heads, dim], k [rows, kv_heads, dim] or None, of one type (float16, bfloat16, float32); the elements
    of a head lie side by side, rows and heads may have any stride.  positions: float32 or int32 [rows, axes];
    freqs float32 [pairs], axes int32 [pairs]: pair i turns by positions[:, axes[i]] * freqs[i].  q_weight,
    k_weight: [dim] of q's type, or None for no norm.  n_items (int32 on the GPU): rows from n_items * item_rows
    on are left as they were.  out: (q_out, k_out), which may be (q, k).  Returns (q_out, k_out)."""
    import torch
    where = "norm_rotate"
    _need(q.is_cuda and q.dim() == 3 and str(q.dtype) in _DTYPES, where, "q is not a CUDA tensor [rows, heads, dim]")
    dev, (rows, heads, dim) = q.device, q.shape
    kv = 0 if k is None else k.shape[1]
    _need(k is None or (k.dim() == 3 and k.shape[0] == rows and k.shape[2] == dim and k.dtype == q.dtype), where,
          "k does not fit q")
    if out is None:
        out = (torch.empty((rows, heads, dim), dtype=q.dtype, device=dev),
               None if k is None else torch.empty((rows, kv, dim), dtype=q.dtype, device=dev))
    q_out, k_out = out
    for name, a, b in (("q", q, q_out), ("k", k, k_out)):
        if a is None:
            continue
        _need(b is not None and b.shape == a.shape and b.dtype == a.dtype, where, f"the output of {name} has another shape")
        _need(dim == 1 or (a.stride(2) == 1 and b.stride(2) == 1), where, f"the elements of a head of {name} are apart")
    for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
        _need(w is None or (w.shape == (dim,) and w.dtype == q.dtype and w.is_contiguous()), where,
              f"{name} is not a contiguous vector [dim] of q's type")
    _need(freqs.dim() == 1 and freqs.dtype == torch.float32 and freqs.is_contiguous(), where, "freqs is not a float32 vector")
    pairs = freqs.numel()
    _int32_vector(where, "axes", axes, pairs)
    _int32_vector(where, "n_items", n_items, 1)
    _need(positions.dim() == 2 and positions.shape[0] == rows and positions.is_contiguous()
          and positions.dtype in (torch.float32, torch.int32), where, "positions is not a contiguous float32 or int32 [rows, axes]")
    _on_device(where, dev, k=k, positions=positions, freqs=freqs, axes=axes, q_weight=q_weight, k_weight=k_weight,
               n_items=n_items, q_out=q_out, k_out=k_out)
    a = B.Rotate()
    a.device, a.dtype, a.heads, a.kv_heads, a.head_dim, a.pairs = dev.index, _DTYPES[str(q.dtype)], heads, kv, dim, pairs
    a.interleaved, a.num_axes = 1 if interleaved else 0, positions.shape[1]
    a.positions_are_int = 1 if positions.dtype == torch.int32 else 0
    a.rows, a.eps = rows, eps
    a.q, a.q_out = _heads(q), _heads(q_out)
    if k is not None:
        a.k, a.k_out = _heads(k), _heads(k_out)
    a.d_q_weight = None if q_weight is None else q_weight.data_ptr()
    a.d_k_weight = None if k_weight is None else k_weight.data_ptr()
    a.d_positions, a.d_freqs, a.d_axes = positions.data_ptr(), freqs.data_ptr(), axes.data_ptr()
    if n_items is not None:
        a.d_n_items, a.item_rows = n_items.data_ptr(), item_rows
    rc = B.load_library().octo_norm_rotate(ctypes.byref(a), _stream_of(torch, dev, stream))
    if rc != B.OCTO_OK:
        raise B.OctoError(rc, "octo_norm_rotate")
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
    import torch
    where = "cross_attention"
    _need(q.is_cuda and q.dim() == 3 and q.dtype in (torch.float16, torch.bfloat16), where,
          "q is not a float16 or bfloat16 CUDA tensor [rows, heads, dim]")
    dev, (q_total, heads, dim) = q.device, q.shape
    _need(k.dim() == 3 and k.shape == v.shape and k.shape[2] == dim and k.dtype == q.dtype and v.dtype == q.dtype, where,
          "k and v do not fit q")
    k_total, kv = k.shape[0], k.shape[1]
    _need(kv > 0 and heads % kv == 0, where, "kv_heads does not divide heads")
    if out is None:
        out = torch.empty((q_total, heads, dim), dtype=q.dtype, device=dev)
    _need(out.shape == q.shape and out.dtype == q.dtype, where, "out has another shape")
    for name, t in (("q", q), ("k", k), ("v", v), ("out", out)):
        _need(dim == 1 or t.stride(2) == 1, where, f"the elements of a head of {name} are apart")
    _int32_vector(where, "q_offsets", q_offsets, segments + 1)
    _int32_vector(where, "k_offsets", k_offsets, segments + 1)
    _need(key_mask is None or (key_mask.dtype in (torch.uint8, torch.bool) and key_mask.shape == (k_total,)
                               and key_mask.is_contiguous()), where, "key_mask is not a contiguous uint8 or bool [k_total]")
    _need(status is None or (status.element_size() == 4 and status.numel() >= 1), where, "status is not a 32-bit word")
    _on_device(where, dev, k=k, v=v, out=out, q_offsets=q_offsets, k_offsets=k_offsets, key_mask=key_mask, status=status)
    a = B.Attend()
    a.device, a.dtype, a.segments, a.heads, a.kv_heads, a.head_dim = dev.index, _DTYPES[str(q.dtype)], segments, heads, kv, dim
    a.q_total, a.k_total = q_total, k_total
    a.q, a.k, a.v, a.out = _heads(q), _heads(k), _heads(v), _heads(out)
    a.d_q_offsets = None if q_offsets is None else q_offsets.data_ptr()
    a.d_k_offsets = None if k_offsets is None else k_offsets.data_ptr()
    a.q_rows, a.k_rows, a.q_first, a.k_first = q_rows, k_rows, q_first, k_first
    a.max_q, a.max_k = max_q or 0, max_k or 0
    a.d_key_mask = None if key_mask is None else key_mask.data_ptr()
    a.scale = dim ** -0.5 if scale is None else scale
    a.d_status = None if status is None else status.data_ptr()
    lib, raw = B.load_library(), _stream_of(torch, dev, stream)
    need = ctypes.c_int64(0)
    rc = lib.octo_attend_workspace(ctypes.byref(a), ctypes.byref(need))
    if rc != B.OCTO_OK:
        raise B.OctoError(rc, "octo_attend_workspace")
    workspace = None
    if need.value:
        workspace = torch.empty((need.value,), dtype=torch.uint8, device=dev)
        if stream is not None:
            workspace.record_stream(stream)
    rc = lib.octo_cross_attention(ctypes.byref(a), None if workspace is None else workspace.data_ptr(), need.value, raw)
    if rc != B.OCTO_OK:
        raise B.OctoError(rc, "octo_cross_attention")
    return out
