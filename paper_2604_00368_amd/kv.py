"""Paged key/value caches as tensors: append, pack, read and attend.

The operators behind ``tent_kv_*`` (include/tent.h) with torch tensors for their device memory: ``Cache`` describes the
pools, ``Batch`` the sequences of a step, and the functions check their tensors, allocate what they return and enqueue on
the current stream.  Nothing is kept between calls; a ``Cache`` and a ``Batch`` hold their tensors alive and can be used
for every layer and step that has the same ones.

With `stream` (a torch.cuda.Stream, or a HIP stream's handle) a call allocates and enqueues there instead.  What it takes
and what it returns is kept from being allocated again before both streams are done with it; that its inputs are ready
when `stream` gets to it, and its outputs before they are used elsewhere, is for the caller to order.

There is no backward pass.  A tensor that requires gradients is refused while they are recorded (not under torch.no_grad()).

A cache of 16 bits is two tensors [pages, page_tokens, kv_heads, head_dim] of bfloat16 or float16; one of 4 bits is two
uint8 tensors [pages, bytes] (``packed_pool``), whose pages hold 32 values to a shared power of two.  Pages are contiguous
byte ranges either way, so the engine moves them as extents of ``page_bytes``.
"""
from __future__ import annotations

import ctypes as C
import math

import torch

from . import binding as T

_TYPES = {torch.bfloat16: T.TENT_BF16, torch.float16: T.TENT_FP16}
_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else None
_current_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else torch.cuda.current_device


def _stream(index):
    return C.c_void_p(_raw_stream(index) if _raw_stream else torch.cuda.current_stream(index).cuda_stream)


def _on(device, stream, used, call):
    """`call()` with the tensors' device current, as the library launches on that, and with `stream`, if one is given, as the
    current stream, so that what it allocates belongs to the stream that uses it.  The allocator is told that `stream` uses the
    caller's tensors `used`, and that the caller's stream uses what the call has made."""
    if stream is None:
        with torch.cuda.device(device):
            return call()
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(getattr(stream, "cuda_stream", stream)), device=device)
    if stream.device != device:
        raise ValueError(f"stream is on {stream.device}, the tensors on {device}")
    caller = torch.cuda.current_stream(device)
    if stream == caller and _current_device() == device.index:
        return call()
    with torch.cuda.stream(stream):
        for x in used:                                                   # what is no tensor of this device the call refuses
            if isinstance(x, torch.Tensor) and x.device == device:
                x.record_stream(stream)
        result = call()
    for x in result if isinstance(result, tuple) else (result,):
        if x is not None and not any(x is y for y in used):
            x.record_stream(caller)
    return result


def _no_gradients(tensor, name):
    if tensor.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name} requires gradients, and there is no backward pass: detach it, or call under torch.no_grad()")


def _on_gpu(tensor, name, dtype, shape=None):
    if not isinstance(tensor, torch.Tensor) or not tensor.is_cuda:
        raise ValueError(f"{name} must be a tensor on a GPU")
    _no_gradients(tensor, name)
    if tensor.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, not {tensor.dtype}")
    if shape is not None and tuple(tensor.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(tensor.shape)}")
    return tensor


def _rows(tensor, name, dtype, rows, heads, dim, device):
    """A tensor [rows, heads, dim] whose heads are contiguous; its stride from row to row."""
    if type(tensor) is not torch.Tensor:
        _on_gpu(tensor, name, dtype)
    if tensor.dtype is not dtype or tensor.device != device:
        raise ValueError(f"{name} must be {dtype} on {device}, not {tensor.dtype} on {tensor.device}")
    if tensor.shape != (rows, heads, dim):
        raise ValueError(f"{name} must have shape {(rows, heads, dim)}, not {tuple(tensor.shape)}")
    if tensor.requires_grad:
        _no_gradients(tensor, name)
    stride = tensor.stride()
    if (stride[2] != 1 and dim > 1) or (stride[1] != dim and heads > 1):
        raise ValueError(f"{name} must have contiguous heads (strides {stride})")
    return stride[0] if rows > 1 else heads * dim


def _check(status, where):
    if status != T.TENT_OK:
        raise T.TentError(status, where)


def packed_page_bytes(page_tokens: int, kv_heads: int, head_dim: int) -> int:
    """Bytes of a 4-bit page of K or of V."""
    n = T.tent_kv_packed_page(page_tokens, kv_heads, head_dim)
    if not n:
        raise ValueError(f"no 4-bit pages of {page_tokens} tokens, {kv_heads} heads of {head_dim}")
    return n


def packed_pool(n_pages: int, page_tokens: int, kv_heads: int, head_dim: int, device="cuda") -> torch.Tensor:
    """A pool of 4-bit pages of zeros (K and V have one each)."""
    return torch.zeros(n_pages, packed_page_bytes(page_tokens, kv_heads, head_dim), dtype=torch.uint8, device=device)


def rope_table(n_positions: int, rope_dim: int, base: float = 10000.0, device="cuda") -> torch.Tensor:
    """Cosines and sines [n_positions, rope_dim] of angles position * base ** (-2 i / rope_dim), computed in 64 bits."""
    half = rope_dim // 2
    rate = float(base) ** (-torch.arange(half, dtype=torch.float64, device=device) / half)
    angle = torch.arange(n_positions, dtype=torch.float64, device=device)[:, None] * rate
    return torch.cat([angle.cos(), angle.sin()], 1).float()


class Cache:
    """The pools of one layer's keys and values.

    16 bits: Cache(k, v).  4 bits: Cache(k, v, dtype=, page_tokens=, kv_heads=, head_dim=), where `dtype` is the 16-bit type
    of the rows that go in and come out."""

    def __init__(self, k, v, dtype=None, page_tokens=None, kv_heads=None, head_dim=None):
        if not isinstance(k, torch.Tensor) or not isinstance(v, torch.Tensor) or not k.is_cuda or k.device != v.device:
            raise ValueError("k and v must be tensors on one GPU")
        if k.dtype != v.dtype or k.shape != v.shape or k.stride() != v.stride():
            raise ValueError("k and v must have the same type, shape and strides")
        _no_gradients(k, "k")
        _no_gradients(v, "v")
        if k.dtype == torch.uint8:
            if k.dim() != 2 or dtype not in _TYPES or None in (page_tokens, kv_heads, head_dim):
                raise ValueError("a 4-bit cache is uint8 [pages, bytes], with dtype, page_tokens, kv_heads and head_dim")
            if k.shape[1] < packed_page_bytes(page_tokens, kv_heads, head_dim) or k.stride(1) != 1:
                raise ValueError("pages are too short, or not contiguous")
            bits, stride = 4, k.stride(0)
        else:
            if k.dtype not in _TYPES or k.dim() != 4 or dtype not in (None, k.dtype):
                raise ValueError("a 16-bit cache is bfloat16 or float16 [pages, page_tokens, kv_heads, head_dim]")
            dtype, (_, page_tokens, kv_heads, head_dim) = k.dtype, k.shape
            if k[:1].numel() == 0 or not k[0].is_contiguous():
                raise ValueError("pages must be contiguous, not empty, and one at least")
            bits, stride = 16, 2 * k.stride(0)
        if k.shape[0] == 0:
            raise ValueError("a cache needs a page")
        if k.shape[0] == 1:                                              # the stride of one page may be anything
            stride = packed_page_bytes(page_tokens, kv_heads, head_dim) if bits == 4 else 2 * k[0].numel()
        self.k, self.v, self.dtype, self.bits, self.device = k, v, dtype, bits, k.device
        self.page_tokens, self.kv_heads, self.head_dim = int(page_tokens), int(kv_heads), int(head_dim)
        self.c = T.tent_kv_cache(k.data_ptr(), v.data_ptr(), k.shape[0], stride, self.page_tokens, self.kv_heads, self.head_dim,
                                 _TYPES[dtype], bits, 0)
        self.ref = C.byref(self.c)                                       # made once: calls take it as it is
        self.tensors, self.index = (k, v), k.device.index

    @property
    def page_bytes(self) -> int:
        """Bytes of a page of K or of V, as the engine moves it."""
        if self.bits == 4:
            return packed_page_bytes(self.page_tokens, self.kv_heads, self.head_dim)
        return 2 * self.page_tokens * self.kv_heads * self.head_dim


class Batch:
    """The sequences of a step: int32 tensors `page_table` [sequences, pages], `kv_len` [sequences] (with the step's rows) and
    `row_start` [sequences + 1]; `n_rows` rows in all, at most `max_rows` to a sequence, at most `max_kv` tokens each.

    Lengths and page numbers are read on the device.  What is wrong there is left out, and noted in `errors` (an int32 tensor
    of one element, made here) as TENT_KV_BAD_* bits."""

    def __init__(self, page_table, kv_len, row_start, n_rows, max_rows, max_kv):
        _on_gpu(page_table, "page_table", torch.int32)
        if page_table.dim() != 2 or (page_table.shape[1] > 1 and page_table.stride(1) != 1):
            raise ValueError("page_table must be [sequences, pages] with contiguous rows")
        n_seqs = page_table.shape[0]
        for x, name, n in ((kv_len, "kv_len", n_seqs), (row_start, "row_start", n_seqs + 1)):
            if not _on_gpu(x, name, torch.int32, (n,)).is_contiguous() or x.device != page_table.device:
                raise ValueError(f"{name} must be contiguous, on the device of page_table")
        if not (0 <= n_rows < 1 << 31 and 0 <= max_rows < 1 << 31 and 0 <= max_kv < 1 << 31):
            raise ValueError("n_rows, max_rows and max_kv must be 0 or more and below 2^31")
        if n_seqs and n_rows and max_kv > page_table.shape[1] * T.TENT_KV_MAX_PAGE_TOKENS:
            raise ValueError("max_kv does not fit the page table")
        width = page_table.stride(0) if n_seqs > 1 else page_table.shape[1]
        if n_seqs > 1 and width < page_table.shape[1]:
            raise ValueError("rows of page_table overlap")
        self.page_table, self.kv_len, self.row_start, self.device = page_table, kv_len, row_start, page_table.device
        self.n_rows, self.max_kv, self.width = int(n_rows), int(max_kv), page_table.shape[1]
        self.errors = torch.zeros(1, dtype=torch.int32, device=page_table.device)
        self.c = T.tent_kv_batch(page_table.data_ptr(), kv_len.data_ptr(), row_start.data_ptr(), self.errors.data_ptr(), n_seqs, width,
                                 n_rows, max_rows, max_kv, 0)
        self.ref = C.byref(self.c)
        self.tensors = (page_table, kv_len, row_start, self.errors)


def _together(cache, batch):
    if cache.device != batch.device:
        raise ValueError("cache and batch are on different devices")
    if batch.max_kv > batch.width * cache.page_tokens:
        raise ValueError("max_kv does not fit the page table")


def append(cache: Cache, batch: Batch, k, v, q=None, q_weight=None, k_weight=None, eps: float = 1e-6, rope=None, rope_pairs: bool = False,
           positions=None, q_out=None, stream=None):
    """Normalise and rotate `k` (and `q`), write k and v to the pages of the batch's rows, return the queries (or None).

    k, v: [rows, kv_heads, head_dim]; q: [rows, q_heads, head_dim]; all of the cache's type, rows at any stride that is a
    multiple of 8 values.  q_weight, k_weight: [head_dim], RMS norm over a head.  rope: float32 [positions, rope_dim] as
    rope_table makes it, indexed by `positions` (int32 [rows]) or the row's position in its sequence; rope_pairs turns
    neighbouring dimensions instead of halves.  q_out may be q."""
    if stream is not None or cache.index != _current_device():
        return _on(cache.device, stream, (*cache.tensors, *batch.tensors, k, v, q, q_weight, k_weight, rope, positions, q_out),
                   lambda: append(cache, batch, k, v, q, q_weight, k_weight, eps, rope, rope_pairs, positions, q_out))
    _together(cache, batch)
    n, H, D, dtype, device = batch.n_rows, cache.kv_heads, cache.head_dim, cache.dtype, cache.device
    k_stride, v_stride = _rows(k, "k", dtype, n, H, D, device), _rows(v, "v", dtype, n, H, D, device)
    heads = q_stride = q_out_stride = 0
    if q is not None:
        heads = q.shape[1] if isinstance(q, torch.Tensor) and q.dim() == 3 else 0
        q_stride = _rows(q, "q", dtype, n, heads, D, device)
        if q_out is None:
            q_out, q_out_stride = torch.empty((n, heads, D), dtype=dtype, device=device), heads * D
        else:
            q_out_stride = _rows(q_out, "q_out", dtype, n, heads, D, device)
    elif q_out is not None or q_weight is not None:
        raise ValueError("q_out and q_weight go with q")
    for w, name in ((q_weight, "q_weight"), (k_weight, "k_weight")):
        if w is not None and (not _on_gpu(w, name, dtype, (D,)).is_contiguous() or w.device != device):
            raise ValueError(f"{name} must be contiguous, on the cache's device")
    a = T.tent_kv_append_args(q.data_ptr() if q is not None else None, k.data_ptr(), v.data_ptr(), q_out.data_ptr() if q is not None else None,
                              q_stride, k_stride, v_stride, q_out_stride, q_weight.data_ptr() if q_weight is not None else None,
                              k_weight.data_ptr() if k_weight is not None else None)
    a.q_heads, a.eps = heads, eps
    if rope is not None:
        if not _on_gpu(rope, "rope", torch.float32).is_contiguous() or rope.dim() != 2 or rope.device != device:
            raise ValueError("rope must be contiguous [positions, rope_dim] on the cache's device")
        a.rope, a.rope_rows, a.rope_dim, a.flags = rope.data_ptr(), rope.shape[0], rope.shape[1], T.TENT_KV_ROPE_PAIRS if rope_pairs else 0
    if positions is not None:
        if not _on_gpu(positions, "positions", torch.int32, (n,)).is_contiguous() or positions.device != device:
            raise ValueError("positions must be contiguous, on the cache's device")
        a.positions = positions.data_ptr()
    _check(T.lib().tent_kv_append(cache.ref, batch.ref, C.byref(a), _stream(cache.index)), "tent_kv_append")
    return q_out


def pack(src: Cache, dst: Cache, src_pages, dst_pages, errors=None, stream=None):
    """Pack pages src_pages[i] of the 16-bit cache `src` into pages dst_pages[i] of the 4-bit cache `dst` (int32 [pages]).
    `errors`: int32 [1] that page numbers outside the pools are noted in."""
    if stream is not None or src.index != _current_device():
        return _on(src.device, stream, (*src.tensors, *dst.tensors, src_pages, dst_pages, errors), lambda: pack(src, dst, src_pages, dst_pages, errors))
    for x, name in ((src_pages, "src_pages"), (dst_pages, "dst_pages")):
        if not _on_gpu(x, name, torch.int32).is_contiguous() or x.dim() != 1 or x.device != src.device:
            raise ValueError(f"{name} must be contiguous int32 [pages] on the caches' device")
    if src_pages.shape != dst_pages.shape or src.device != dst.device:
        raise ValueError("as many pages on one side as on the other, on one device")
    if errors is not None and _on_gpu(errors, "errors", torch.int32, (1,)).device != src.device:
        raise ValueError("errors must be on the caches' device")
    _check(T.lib().tent_kv_pack(src.ref, dst.ref, src_pages.data_ptr(), dst_pages.data_ptr(), src_pages.shape[0],
                                errors.data_ptr() if errors is not None else None, _stream(src.index)), "tent_kv_pack")


def read(cache: Cache, batch: Batch, k_out=None, v_out=None, stream=None):
    """The keys and values of the batch's rows as dense tensors [rows, kv_heads, head_dim] of the cache's type."""
    if stream is not None or cache.index != _current_device():
        return _on(cache.device, stream, (*cache.tensors, *batch.tensors, k_out, v_out), lambda: read(cache, batch, k_out, v_out))
    _together(cache, batch)
    shape = (batch.n_rows, cache.kv_heads, cache.head_dim)
    if k_out is None:
        k_out = torch.empty(shape, dtype=cache.dtype, device=cache.device)
    if v_out is None:
        v_out = torch.empty(shape, dtype=cache.dtype, device=cache.device)
    stride = _rows(k_out, "k_out", cache.dtype, *shape, cache.device)
    if _rows(v_out, "v_out", cache.dtype, *shape, cache.device) != stride:
        raise ValueError("k_out and v_out must have the same strides")
    _check(T.lib().tent_kv_read(cache.ref, batch.ref, k_out.data_ptr(), v_out.data_ptr(), stride, _stream(cache.index)), "tent_kv_read")
    return k_out, v_out


def attend(cache: Cache, batch: Batch, q, scale: float = None, window: int = 0, causal: bool = True, out=None, want_lse: bool = False,
           workspace=None, stream=None):
    """Attention of the batch's rows over their sequences: [rows, q_heads, head_dim], and with `want_lse` the logsumexp of the
    scores [rows, q_heads] in float32.  scale: 1 / sqrt(head_dim) unless given; window: a row sees its last `window` tokens;
    causal=False: every row sees its whole sequence.  workspace: a contiguous uint8 tensor of at least attend_workspace
    bytes to use instead of a new one."""
    if stream is not None or cache.index != _current_device():
        return _on(cache.device, stream, (*cache.tensors, *batch.tensors, q, out, workspace),
                   lambda: attend(cache, batch, q, scale, window, causal, out, want_lse, workspace))
    _together(cache, batch)
    n, D, dtype, device = batch.n_rows, cache.head_dim, cache.dtype, cache.device
    heads = q.shape[1] if isinstance(q, torch.Tensor) and q.dim() == 3 else 0
    q_stride = _rows(q, "q", dtype, n, heads, D, device)
    if out is None:
        out, out_stride = torch.empty((n, heads, D), dtype=dtype, device=device), heads * D
    else:
        out_stride = _rows(out, "out", dtype, n, heads, D, device)
    if not 0 <= window < 1 << 31:
        raise ValueError("window must be 0 or more and below 2^31")
    lse = torch.empty((n, heads), dtype=torch.float32, device=device) if want_lse else None
    a = T.tent_kv_attend_args(q.data_ptr(), out.data_ptr(), lse.data_ptr() if want_lse else None, q_stride, out_stride, None, 0, heads, window,
                              0 if causal else T.TENT_KV_ATTEND_ALL, 1.0 / math.sqrt(D) if scale is None else scale)
    L, need, ref = T.lib(), C.c_uint64(), C.byref(a)
    _check(L.tent_kv_attend_workspace(cache.ref, batch.ref, ref, C.byref(need)), "tent_kv_attend_workspace")
    if need.value:
        if workspace is None:
            workspace = torch.empty(need.value, dtype=torch.uint8, device=device)
        elif not _on_gpu(workspace, "workspace", torch.uint8).is_contiguous() or workspace.device != device:
            raise ValueError("workspace must be contiguous, on the cache's device")
        a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel()
    _check(L.tent_kv_attend(cache.ref, batch.ref, ref, _stream(cache.index)), "tent_kv_attend")
    return (out, lse) if want_lse else out


def attend_workspace(cache: Cache, batch: Batch, q_heads: int, window: int = 0, causal: bool = True) -> int:
    """Bytes of workspace that attend takes for such a batch."""
    _together(cache, batch)
    return T.tent_kv_attend_workspace(cache.c, batch.c, T.tent_kv_attend_args(q_heads=q_heads, window=window, scale=1.0,
                                                                             flags=0 if causal else T.TENT_KV_ATTEND_ALL))
