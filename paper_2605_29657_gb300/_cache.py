"""What follows pruning: rotary positions with several axes, and a paged
cache held in 8 bits with the calls that fill it, attend over it and manage
its pages (include/occam.h). Argument marshalling only, as in _lib.

stream: the stream a call runs on (default: the current one of its tensors'
device). New results are allocated on that stream; as with every tensor used on
two streams, order them and keep or record (Tensor.record_stream) what the
other one still uses."""

from __future__ import annotations

import ctypes
import struct

import torch

from ._lib import (
    OCCAM_ERR_INVALID_ARG,
    CAppendRopeArgs,
    CAttendArgs,
    CCache,
    CRopeTensor,
    OccamError,
    _check,
    _dev_tensor,
    _ptr,
    library,
)

_DTYPE = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
_ROWS = {torch.bfloat16: 0, torch.float16: 1}  # element types of cache rows
_PAIRING = {"half": 0, "adjacent": 1}
E4M3 = torch.float8_e4m3fn

# occam_rope_tensor and occam_attend_args as packed bytes: a decode step makes
# these calls once a layer, and filling a ctypes structure field by field takes longer
_ROPE_TENSOR = struct.Struct("@PPiqqqq")
_ATTEND_ARGS = struct.Struct("@iiiiqqPPPiiPPfPPq")
_APPEND_ROPE_ARGS = struct.Struct("@iiiiiiqPqPqPPPqPPP")
assert _ROPE_TENSOR.size == ctypes.sizeof(CRopeTensor) and _ATTEND_ARGS.size == ctypes.sizeof(CAttendArgs)
assert _APPEND_ROPE_ARGS.size == ctypes.sizeof(CAppendRopeArgs)


def _bad(msg: str):
    raise OccamError(OCCAM_ERR_INVALID_ARG, msg)


# A call's tensors are all on one GPU, `at` below (its index); the call is made with that one current.

def _on(stream, at: int) -> int:
    """The stream's handle; the device's current one by default."""
    if stream is not None:
        if stream.device.index != at:
            _bad(f"the stream is on {stream.device}, the tensors on cuda:{at}")
        return stream.cuda_stream
    return torch._C._cuda_getCurrentRawStream(at)


def _call(at: int, fn, *args) -> None:
    if torch._C._cuda_getDevice() == at:
        rc = fn(*args)
    else:
        with torch.cuda.device(at):
            rc = fn(*args)
    if rc:
        _check(rc, fn.__name__)


def _empty(shape, dtype, device, stream) -> torch.Tensor:
    """A new result, of the stream that writes it: another stream's freed memory may still be in use there."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _dense(t, dtype, name: str, at: int) -> torch.Tensor:
    if not isinstance(t, torch.Tensor) or t.get_device() != at:
        _bad(f"{name} must be a tensor on cuda:{at}")
    return _dev_tensor(t, dtype, name)


def _rows_tensor(t, name: str, dtypes, at: int, heads: int | None = None, dim: int | None = None) -> torch.Tensor:
    """A CUDA tensor [rows, heads, dim] whose heads are dense; rows may be strided."""
    if not isinstance(t, torch.Tensor) or t.get_device() != at:
        _bad(f"{name} must be a tensor on cuda:{at}")
    if t.dtype not in dtypes:
        _bad(f"{name} must be one of {[str(d) for d in dtypes]}, got {t.dtype}")
    shape = t.shape
    if len(shape) != 3 or (heads is not None and shape[1] != heads) or (dim is not None and shape[2] != dim):
        _bad(f"{name} must be [rows, {heads or 'heads'}, {dim or 'dim'}], got {list(shape)}")
    if not t.is_contiguous():
        _, h, d = t.stride()
        if t.numel() and (d != 1 or (shape[1] > 1 and h != shape[2])):
            _bad(f"{name} must be dense in its last two dimensions")
    return t


def _row_stride(t: torch.Tensor) -> int:
    """Elements from one row to the next (a single row has none: its own size)."""
    return t.stride(0) if t.shape[0] > 1 else t.shape[1] * t.shape[2]


# ------------------------------------------------------------------ rotary positions

def rope_axes(sections, interleaved: bool = False, device="cuda") -> torch.Tensor:
    """The axis of each pair, int32 [sum(sections)]. sections[a] pairs turn
    with axis a: in consecutive runs, or interleaved (pair i with axis i %
    axes as long as that axis has pairs left, then axis 0)."""
    n = sum(sections)
    if not interleaved:
        axis = [a for a, s in enumerate(sections) for _ in range(s)]
    else:
        axis = [0] * n
        for a in range(1, len(sections)):
            for i in range(a, len(sections) * sections[a], len(sections)):
                if i >= n:
                    _bad("an interleaved section reaches past the pairs")
                axis[i] = a
    return torch.tensor(axis, dtype=torch.int32, device=device)


def occam_rope(q, k, positions, inv_freq, axis, pairing: str = "half", inverse: bool = False, out_q=None, out_k=None,
               stream=None):
    """Turns q [rows, heads, dim] and k (None: q alone) by their positions
    [axes, rows] int32: pair i by positions[axis[i]] * inv_freq[i]; pairs are
    (i, i + rot/2) for "half" and (2i, 2i + 1) for "adjacent", rot = 2 *
    len(inv_freq). inverse: by the negative angle, the gradient's map. q and k may be
    strided in rows and heads (views of one projection). Results are new
    dense tensors unless out_q / out_k are given (q itself: in place). Returns (q, k)."""
    if pairing not in _PAIRING:
        _bad(f"pairing must be one of {sorted(_PAIRING)}")
    if not isinstance(q, torch.Tensor) or not q.is_cuda or q.dim() != 3 or q.dtype not in _DTYPE:
        _bad("q must be a CUDA tensor [rows, heads, dim] of bfloat16, float16 or float32")
    rows, _, dim = q.shape
    dtype, at = q.dtype, q.get_device()
    pairs = _turns(positions, inv_freq, axis, rows, at)
    on = _on(stream, at)
    packed, out_q = _rope_tensor(q, out_q, "q", rows, dim, dtype, at, stream)
    n = 1
    if k is not None:
        more, out_k = _rope_tensor(k, out_k, "k", rows, dim, dtype, at, stream)
        packed += more
        n = 2
    elif out_k is not None:
        _bad("out_k without k")
    _call(at, library().occam_rope, _DTYPE[dtype], rows, dim, 2 * pairs, _PAIRING[pairing], int(bool(inverse)),
          positions.data_ptr(), positions.stride(0), positions.shape[0], inv_freq.data_ptr(), axis.data_ptr(), n, packed, on)
    return out_q, out_k


def _turns(positions, inv_freq, axis, rows: int, at: int) -> int:
    """The number of pairs."""
    pairs = _vector(inv_freq, torch.float32, None, "inv_freq", at).shape[0]
    _vector(axis, torch.int32, pairs, "axis", at)
    if not isinstance(positions, torch.Tensor) or positions.get_device() != at or positions.dtype != torch.int32 or \
            positions.dim() != 2 or positions.shape[1] != rows or (rows > 1 and positions.stride(1) != 1):
        _bad(f"positions must be an int32 tensor [axes, rows] on cuda:{at}, dense in rows")
    return pairs


def _rope_tensor(x, out, name, rows, dim, dtype, at, stream):
    if not isinstance(x, torch.Tensor) or x.get_device() != at or x.dtype != dtype or x.dim() != 3 or x.shape[0] != rows or \
            x.shape[2] != dim:
        _bad(f"{name} must be a tensor [{rows}, heads, {dim}] {dtype} on cuda:{at}")
    row, head, one = x.stride()
    if out is None:
        out = _empty(x.shape, dtype, x.device, stream)
        heads = x.shape[1]
        out_row, out_head, out_one = heads * dim, dim, 1
    else:
        if not isinstance(out, torch.Tensor) or out.get_device() != at or out.shape != x.shape or out.dtype != dtype:
            _bad(f"out_{name} must be like {name}")
        heads = x.shape[1]
        out_row, out_head, out_one = out.stride()
    if (one != 1 or out_one != 1) and x.numel():
        _bad(f"{name} must be dense in its last dimension")
    return _ROPE_TENSOR.pack(x.data_ptr(), out.data_ptr(), heads, row, head, out_row, out_head), out


# ------------------------------------------------------------------ the cache

class PagedCache:
    """A pool of pages for `layers` layers, held as e4m3 codes with an fp32
    scale per (layer, page, head), and the tables of `max_seqs` sequences.

    k, v [layers, pages, heads, page_tokens, dim] float8_e4m3fn; k_scale,
    v_scale [layers, pages, heads]; table [max_seqs, max_pages] int32 (-1: no
    page); length [max_seqs]; refs [pages]. One workspace (ws) serves one
    call at a time: for calls in flight on several streams give each its own
    (alloc_workspace)."""

    def __init__(self, layers: int, pages: int, heads: int, dim: int, max_seqs: int, max_pages: int,
                 page_tokens: int = 64, max_tokens: int | None = None, device="cuda"):
        shape = (layers, pages, heads, page_tokens, dim)
        self._set(torch.zeros(shape, dtype=torch.uint8, device=device).view(E4M3),
                  torch.zeros(shape, dtype=torch.uint8, device=device).view(E4M3),
                  torch.ones(shape[:3], dtype=torch.float32, device=device),
                  torch.ones(shape[:3], dtype=torch.float32, device=device),
                  torch.full((max_seqs, max_pages), -1, dtype=torch.int32, device=device),
                  torch.zeros(max_seqs, dtype=torch.int32, device=device),
                  torch.zeros(pages, dtype=torch.int32, device=device), max_tokens)

    @classmethod
    def wrap(cls, k, v, k_scale, v_scale, table, length, refs, max_tokens: int | None = None) -> "PagedCache":
        """A cache over existing tensors (nothing is copied)."""
        self = cls.__new__(cls)
        self._set(k, v, k_scale, v_scale, table, length, refs, max_tokens)
        return self

    def _set(self, k, v, k_scale, v_scale, table, length, refs, max_tokens):
        at = _dev_tensor(k, E4M3, "k").get_device()
        _dense(v, E4M3, "v", at)
        _dense(k_scale, torch.float32, "k_scale", at); _dense(v_scale, torch.float32, "v_scale", at)
        _dense(table, torch.int32, "table", at); _dense(length, torch.int32, "length", at)
        _dense(refs, torch.int32, "refs", at)
        if k.dim() != 5 or v.shape != k.shape or k_scale.shape != k.shape[:3] or v_scale.shape != k.shape[:3]:
            _bad("k and v must be [layers, pages, heads, page_tokens, dim], their scales [layers, pages, heads]")
        if table.dim() != 2 or length.shape != table.shape[:1] or refs.shape != k.shape[1:2]:
            _bad("table must be [max_seqs, max_pages], length [max_seqs], refs [pages]")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.table, self.length, self.refs = table, length, refs
        self.layers, self.pages, self.heads, self.page_tokens, self.dim = k.shape
        self.max_seqs, self.max_pages = table.shape
        # flags one compact call may pass: by default a token of every page of the pool
        self.max_tokens = self.pages * self.page_tokens if max_tokens is None else int(max_tokens)
        self.device, self.at = k.device, at
        self._c = CCache(self.layers, self.pages, self.heads, self.dim, self.page_tokens, self.max_seqs, self.max_pages,
                         _ptr(k), _ptr(v), _ptr(k_scale), _ptr(v_scale), _ptr(table), _ptr(length), _ptr(refs))
        self._ref = ctypes.byref(self._c)
        self.ws = self.alloc_workspace()
        self._ws = (self.ws.data_ptr(), self.ws.numel())

    def alloc_workspace(self, rows: int = 0, heads: int = 0) -> torch.Tensor:
        """A workspace of the cache calls, zero-filled and 256-byte aligned. rows, heads: the most
        query rows and heads of an occam_cache_attend_shared call with it (0: it serves none)."""
        n = ctypes.c_size_t(0)
        _check(library().occam_cache_workspace_size(self._ref, self.max_tokens, ctypes.byref(n)),
               "occam_cache_workspace_size")
        size = n.value
        if rows:
            _check(library().occam_cache_shared_workspace_size(self._ref, int(rows), int(heads), ctypes.byref(n)),
                   "occam_cache_shared_workspace_size")
            size = max(size, n.value)
        ws = torch.zeros(size + 256, dtype=torch.uint8, device=self.device)
        off = (-ws.data_ptr()) % 256
        return ws[off:off + size]

    def status(self, stream=None, ws=None) -> int:
        """Reads and clears the status word (synchronises the stream)."""
        v = ctypes.c_int32(0)
        _call(self.at, library().occam_get_status, _workspace(self, ws)[0], ctypes.byref(v), _on(stream, self.at))
        return int(v.value)


def _workspace(cache, ws):
    if not isinstance(cache, PagedCache):
        _bad("cache must be a PagedCache")
    if ws is None:
        return cache._ws
    _dense(ws, torch.uint8, "ws", cache.at)
    return ws.data_ptr(), ws.numel()


def _vector(t, dtype, n: int | None, name: str, at: int) -> torch.Tensor:
    if not isinstance(t, torch.Tensor) or t.get_device() != at or t.dtype != dtype or t.dim() != 1 or \
            (n is not None and t.shape[0] != n) or not t.is_contiguous():
        _bad(f"{name} must be a dense vector of {dtype} on cuda:{at}" + ("" if n is None else f" with {n} entries"))
    return t


def occam_cache_extend(cache: PagedCache, seqs, counts, ws=None, stream=None) -> None:
    """Sequence seqs[i] grows by counts[i] tokens: pages are taken and lengths raised. After a
    call that recorded an error, extend and append with that workspace do nothing until status() is read."""
    wp, wn = _workspace(cache, ws)
    n = _vector(seqs, torch.int32, None, "seqs", cache.at).shape[0]
    _vector(counts, torch.int32, n, "counts", cache.at)
    _call(cache.at, library().occam_cache_extend, cache._ref, n, _ptr(seqs), _ptr(counts), wp, wn, _on(stream, cache.at))


def occam_cache_append(cache: PagedCache, layer: int, k, v, seqs, row_off, ws=None, stream=None) -> None:
    """Writes rows row_off[i] .. row_off[i+1] of k and v [rows, heads, dim]
    (bfloat16 or float16, rows may be strided) as the last tokens of sequence
    seqs[i] in one layer. Pages that other sequences hold too are not written."""
    wp, wn = _workspace(cache, ws)
    _rows_tensor(k, "k", _ROWS, cache.at, cache.heads, cache.dim)
    _rows_tensor(v, "v", (k.dtype,), cache.at, cache.heads, cache.dim)
    if v.shape[0] != k.shape[0]:
        _bad("k and v must have as many rows")
    n = _vector(seqs, torch.int32, None, "seqs", cache.at).shape[0]
    _vector(row_off, torch.int64, n + 1, "row_off", cache.at)
    _call(cache.at, library().occam_cache_append, cache._ref, int(layer), _DTYPE[k.dtype], k.shape[0], _ptr(k), _row_stride(k),
          _ptr(v), _row_stride(v), n, _ptr(seqs), _ptr(row_off), wp, wn, _on(stream, cache.at))


def occam_cache_append_rope(cache: PagedCache, layer: int, q, k, v, seqs, row_off, positions, inv_freq, axis,
                            pairing: str = "half", out_q=None, ws=None, stream=None):
    """occam_cache_append with the keys turned by their positions (as occam_rope, in fp32 until they
    are rounded to codes) and the queries q [rows, heads, dim] (None: none) of the same rows
    turned beside them. Returns the turned queries: a new dense tensor unless out_q is given (q
    itself: in place)."""
    wp, wn = _workspace(cache, ws)
    if pairing not in _PAIRING:
        _bad(f"pairing must be one of {sorted(_PAIRING)}")
    _rows_tensor(k, "k", _ROWS, cache.at, cache.heads, cache.dim)
    _rows_tensor(v, "v", (k.dtype,), cache.at, cache.heads, cache.dim)
    rows = k.shape[0]
    if v.shape[0] != rows:
        _bad("k and v must have as many rows")
    n = _vector(seqs, torch.int32, None, "seqs", cache.at).shape[0]
    _vector(row_off, torch.int64, n + 1, "row_off", cache.at)
    pairs = _turns(positions, inv_freq, axis, rows, cache.at)
    on = _on(stream, cache.at)
    packed = None
    if q is not None:
        packed, out_q = _rope_tensor(q, out_q, "q", rows, cache.dim, k.dtype, cache.at, stream)
    elif out_q is not None:
        _bad("out_q without q")
    try:
        a = CAppendRopeArgs.from_buffer_copy(_APPEND_ROPE_ARGS.pack(
            layer, _ROWS[k.dtype], n, 2 * pairs, _PAIRING[pairing], positions.shape[0], rows, k.data_ptr(), _row_stride(k), v.data_ptr(),
            _row_stride(v), seqs.data_ptr(), row_off.data_ptr(), positions.data_ptr(), positions.stride(0), inv_freq.data_ptr(),
            axis.data_ptr(), 0))
    except struct.error as e:
        _bad(f"layer: {e}")
    if packed is not None:
        a.q = packed
    _call(cache.at, library().occam_cache_append_rope, cache._ref, ctypes.byref(a), wp, wn, on)
    return out_q


def _attend_args(cache, layer, q, seqs, row_off, max_rows, scale, causal, keep, keep_off, out, lse, stream):
    """(packed arguments, out, lse, stream handle) of an attention call."""
    _rows_tensor(q, "q", _ROWS, cache.at, None, cache.dim)
    rows, heads, dim = q.shape
    n = _vector(seqs, torch.int32, None, "seqs", cache.at).shape[0]
    _vector(row_off, torch.int64, n + 1, "row_off", cache.at)
    total_keep = 0
    if keep is not None:
        _dense(keep, torch.uint8, "keep", cache.at)
        if keep_off is None:
            _bad("keep needs keep_off")
        _vector(keep_off, torch.int64, n + 1, "keep_off", cache.at)
        total_keep = keep.numel()
    on = _on(stream, cache.at)
    if out is None:
        out = _empty((rows, heads, dim), q.dtype, q.device, stream)
    elif _dense(out, q.dtype, "out", cache.at).shape != q.shape:
        _bad("out must be like q")
    if lse is None:
        lse = _empty((rows, heads), torch.float32, q.device, stream)
    elif _dense(lse, torch.float32, "lse", cache.at).shape != q.shape[:2]:
        _bad("lse must be [rows, heads]")
    try:
        a = _ATTEND_ARGS.pack(layer, _ROWS[q.dtype], heads, 1 if causal else 0, rows, _row_stride(q), q.data_ptr(),
                              out.data_ptr(), lse.data_ptr(), n, max_rows, seqs.data_ptr(), row_off.data_ptr(), scale,
                              0 if keep is None else keep.data_ptr(), 0 if keep is None else keep_off.data_ptr(),
                              total_keep)
    except struct.error as e:
        _bad(f"layer, max_rows or scale: {e}")
    return a, out, lse, on


def occam_cache_attend(cache: PagedCache, layer: int, q, seqs, row_off, max_rows: int, scale: float = 0.0,
                       causal: bool = True, keep=None, keep_off=None, out=None, lse=None, ws=None, stream=None):
    """Attention of the rows of q [rows, heads, dim] (the last tokens of their
    sequences; rows may be strided) over the cache. max_rows: the most rows of one
    sequence. scale 0: 1 / sqrt(dim). keep / keep_off: uint8 flags that hide
    tokens. Returns (out, lse [rows, heads] natural logarithm)."""
    wp, wn = _workspace(cache, ws)
    a, out, lse, on = _attend_args(cache, layer, q, seqs, row_off, max_rows, scale, causal, keep, keep_off, out, lse, stream)
    _call(cache.at, library().occam_cache_attend, cache._ref, a, wp, wn, on)
    return out, lse


def occam_cache_attend_shared(cache: PagedCache, layer: int, q, seqs, row_off, max_rows: int, group_off, max_group_rows: int, ws,
                              scale: float = 0.0, causal: bool = True, out=None, lse=None, stream=None):
    """occam_cache_attend for sequences that share leading pages (forks): group g is seqs[group_off[g]]
    .. seqs[group_off[g + 1] - 1] (int32, from 0 up to the number of sequences), and the full pages that its
    sequences have in common are read once for all their rows, where that saves time. max_group_rows: the most rows of one group.
    ws: alloc_workspace(rows, heads). Returns (out, lse) as occam_cache_attend."""
    wp, wn = _workspace(cache, ws)
    a, out, lse, on = _attend_args(cache, layer, q, seqs, row_off, max_rows, scale, causal, None, None, out, lse, stream)
    groups = _vector(group_off, torch.int32, None, "group_off", cache.at).shape[0] - 1
    if groups < 0:
        _bad("group_off must have an entry more than there are groups")
    try:
        _call(cache.at, library().occam_cache_attend_shared, cache._ref, a, group_off.data_ptr(), groups, max_group_rows, wp, wn, on)
    except ctypes.ArgumentError as e:
        _bad(f"max_group_rows: {e}")
    return out, lse


def occam_cache_fork(cache: PagedCache, src, dst, ws=None, stream=None) -> None:
    """Sequence dst[i] (empty) becomes a copy of src[i]; full pages are shared."""
    wp, wn = _workspace(cache, ws)
    n = _vector(src, torch.int32, None, "src", cache.at).shape[0]
    _vector(dst, torch.int32, n, "dst", cache.at)
    _call(cache.at, library().occam_cache_fork, cache._ref, n, _ptr(src), _ptr(dst), wp, wn, _on(stream, cache.at))


def occam_cache_compact(cache: PagedCache, seqs, keep, keep_off, layers: tuple[int, int] | None = None, ws=None,
                        stream=None) -> None:
    """Keeps the tokens of each sequence whose flag keep[keep_off[i] + p] is
    set (and those past the flags), in order; layers: the range of layers whose
    codes move (default: all)."""
    wp, wn = _workspace(cache, ws)
    n = _vector(seqs, torch.int32, None, "seqs", cache.at).shape[0]
    _dense(keep, torch.uint8, "keep", cache.at)
    _vector(keep_off, torch.int64, n + 1, "keep_off", cache.at)
    l0, l1 = (0, cache.layers) if layers is None else layers
    _call(cache.at, library().occam_cache_compact, cache._ref, int(l0), int(l1), n, _ptr(seqs), _ptr(keep), _ptr(keep_off),
          keep.numel(), wp, wn, _on(stream, cache.at))


def occam_cache_release(cache: PagedCache, seqs, ws=None, stream=None) -> None:
    """Empties sequences; their pages lose a reference."""
    wp, wn = _workspace(cache, ws)
    n = _vector(seqs, torch.int32, None, "seqs", cache.at).shape[0]
    _call(cache.at, library().occam_cache_release, cache._ref, n, _ptr(seqs), wp, wn, _on(stream, cache.at))
