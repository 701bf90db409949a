"""Attention of whole prompts: packed sequences of 16-bit rows, and the gradient
(include/occam.h). Argument marshalling only, as in _lib. Streams and new
results as in _cache."""

from __future__ import annotations

import ctypes
import struct

import torch

from ._cache import _DTYPE, _ROWS, _bad, _call, _dense, _empty, _on, _row_stride, _rows_tensor, _vector
from ._lib import CPromptArgs, CPromptGrads, _check, library

# occam_prompt_args as packed bytes (as in _cache)
_PROMPT_ARGS = struct.Struct("@iiiiiiqqPPPqqqPPf0q")
assert _PROMPT_ARGS.size == ctypes.sizeof(CPromptArgs)


def alloc_prompt_workspace(rows: int, heads: int, keys: int | None = None, kv_heads: int | None = None, device="cuda") -> torch.Tensor:
    """A workspace (zero-filled, 256-byte aligned) of occam_prompt_attend and its gradient for up to `rows`
    query rows of `heads` heads and `keys` (None: as many as rows) keys of `kv_heads` (None: heads). One workspace
    serves one call at a time."""
    n = ctypes.c_size_t(0)
    _check(library().occam_prompt_workspace_size(int(rows), int(rows if keys is None else keys), int(heads),
                                                 int(heads if kv_heads is None else kv_heads), ctypes.byref(n)),
           "occam_prompt_workspace_size")
    ws = torch.zeros(n.value + 256, dtype=torch.uint8, device=device)
    off = (-ws.data_ptr()) % 256
    return ws[off:off + n.value]


def _inputs(q, k, v, row_off, key_off, scale, causal):
    if not isinstance(q, torch.Tensor) or not q.is_cuda:
        _bad("q must be a CUDA tensor [rows, heads, dim]")
    at = q.get_device()
    _rows_tensor(q, "q", _ROWS, at)
    rows, heads, dim = q.shape
    _rows_tensor(k, "k", (q.dtype,), at, None, dim)
    _rows_tensor(v, "v", (q.dtype,), at, k.shape[1], dim)
    if v.shape[0] != k.shape[0]:
        _bad("k and v must have as many rows")
    if key_off is None:
        key_off = row_off
    n = _vector(row_off, torch.int64, None, "row_off", at).shape[0] - 1
    if n < 0:
        _bad("row_off must have an entry more than there are sequences")
    _vector(key_off, torch.int64, n + 1, "key_off", at)
    try:
        return at, _PROMPT_ARGS.pack(_DTYPE[q.dtype], heads, k.shape[1], dim, 1 if causal else 0, n, rows, k.shape[0], q.data_ptr(),
                                     k.data_ptr(), v.data_ptr(), _row_stride(q), _row_stride(k), _row_stride(v),
                                     row_off.data_ptr(), key_off.data_ptr(), scale)
    except (struct.error, OverflowError) as e:
        _bad(f"scale or a size: {e}")


def occam_prompt_attend(q, k, v, row_off, ws, key_off=None, scale: float = 0.0, causal: bool = True, out=None, lse=None,
                        stream=None):
    """Attention of packed sequences: rows row_off[i] .. row_off[i+1] of q [rows,
    heads, dim] over rows key_off[i] .. key_off[i+1] (None: the same) of k and v [keys,
    kv_heads, dim] (bfloat16 or float16; rows may be strided). causal: the queries are the
    last of their sequence's tokens. scale 0: 1 / sqrt(dim). ws: alloc_prompt_workspace. Returns
    (out, lse [rows, heads] natural logarithm); rows that belong to no sequence are not written."""
    at, args = _inputs(q, k, v, row_off, key_off, scale, causal)
    _dense(ws, torch.uint8, "ws", at)
    on = _on(stream, at)
    if out is None:
        out = _empty(q.shape, q.dtype, q.device, stream)
    elif _dense(out, q.dtype, "out", at).shape != q.shape:
        _bad("out must be like q")
    if lse is None:
        lse = _empty(q.shape[:2], torch.float32, q.device, stream)
    elif _dense(lse, torch.float32, "lse", at).shape != q.shape[:2]:
        _bad("lse must be [rows, heads]")
    _call(at, library().occam_prompt_attend, args, out.data_ptr(), lse.data_ptr(), ws.data_ptr(), ws.numel(), on)
    return out, lse


def occam_prompt_attend_grad(q, k, v, out, lse, dout, row_off, ws, key_off=None, scale: float = 0.0, causal: bool = True, dq=None,
                             dk=None, dv=None, stream=None):
    """The gradient of occam_prompt_attend: from its arguments, its results out and lse, and dout [rows, heads, dim], a
    loss's gradient with respect to out (rows may be strided). Returns (dq, dk, dv), new dense tensors unless
    given (their rows may be strided: views of one projection's gradient). Rows and keys that belong to no
    sequence are not written: give zeroed tensors where some are padded."""
    at, args = _inputs(q, k, v, row_off, key_off, scale, causal)
    _dense(ws, torch.uint8, "ws", at)
    on = _on(stream, at)
    if _dense(out, q.dtype, "out", at).shape != q.shape:
        _bad("out must be like q")
    if _dense(lse, torch.float32, "lse", at).shape != q.shape[:2]:
        _bad("lse must be [rows, heads]")
    _rows_like(dout, q, "dout", at)
    grads = []
    for name, given, like in (("dq", dq, q), ("dk", dk, k), ("dv", dv, v)):
        if given is None:
            given = _empty(like.shape, like.dtype, like.device, stream)
        else:
            _rows_like(given, like, name, at)
        grads.append(given)
    dq, dk, dv = grads
    g = CPromptGrads(out.data_ptr(), lse.data_ptr(), dout.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), _row_stride(dout),
                     _row_stride(dq), _row_stride(dk), _row_stride(dv))
    _call(at, library().occam_prompt_attend_grad, args, ctypes.byref(g), ws.data_ptr(), ws.numel(), on)
    return dq, dk, dv


def _rows_like(t, like, name: str, at: int) -> None:
    if _rows_tensor(t, name, (like.dtype,), at, like.shape[1], like.shape[2]).shape[0] != like.shape[0]:
        _bad(f"{name} must have {like.shape[0]} rows")
