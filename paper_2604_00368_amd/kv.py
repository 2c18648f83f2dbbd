"""Paged key/value caches as tensors: append, pack, read and attend; verify, weigh, choose and keep.

The operators behind ``tent_kv_*`` (include/tent.h) with torch tensors for their device memory: ``Cache`` describes the
pools, ``Batch`` the sequences of a step, and the functions check their tensors, allocate what they return and enqueue on
the current stream.  Nothing is kept between calls; a ``Cache`` and a ``Batch`` hold their tensors alive and can be used
for every layer and step that has the same ones.

With `stream` (a torch.cuda.Stream, or a HIP stream's handle) a call allocates and enqueues there instead.  What it takes
and what it returns is kept from being allocated again before both streams are done with it; that its inputs are ready
when `stream` gets to it, and its outputs before they are used elsewhere, is for the caller to order.

There is no backward pass.  A tensor that requires gradients is refused while they are recorded (not under torch.no_grad()).

Speculative decoding: append the drafted tokens behind the last decided one, attend with tree= (``tree_masks``), verify, keep
with rows=True.  Eviction: weigh after attention, choose, keep.

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


def tree_masks(parents, row_start, max_rows: int):
    """What attend's `tree` takes for a tree: bits [rows, words] (int64) of the rows that each row sees, itself and those on the way
    to it, and how far down each row is [rows] (int32; what to add to the context's length for its position).

    parents: int32 [rows], the row of its sequence that a row is behind (verify's); a row that is behind none before it is a
    root.  row_start: int32 [sequences + 1]."""
    n, words, device = parents.shape[0], max(1, -(-max_rows // 64)), parents.device
    row = torch.arange(n, device=device)
    first = row_start.long()[torch.bucketize(row, row_start[1:].long(), right=True).clamp(max=max(row_start.shape[0] - 2, 0))]
    local = row - first
    up = torch.where((parents >= 0) & (parents < local), first + parents, -1)            # the row above, then the one 2, 4, .. up
    bit = torch.ones((), dtype=torch.int64, device=device) << (local & 63)
    masks = torch.where(torch.arange(words, device=device) == (local >> 6)[:, None], bit[:, None], 0)
    reach = torch.ones(n, dtype=torch.int32, device=device)
    for _ in range(max(max_rows - 1, 0).bit_length()):
        there = up >= 0
        at = up.clamp(min=0)
        masks = masks | torch.where(there[:, None], masks[at], 0)
        reach = reach + torch.where(there, reach[at], 0)
        up = torch.where(there, up[at], -1)
    return masks, reach - 1


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
           workspace=None, stream=None, tree=None):
    """Attention of the batch's rows over their sequences: [rows, q_heads, head_dim], and with `want_lse` the logsumexp of the
    scores [rows, q_heads] in float32.  scale: 1 / sqrt(head_dim) unless given; window: a row sees its last `window` tokens;
    causal=False: every row sees its whole sequence.  workspace: a contiguous uint8 tensor of at least attend_workspace
    bytes to use instead of a new one.  tree: int64 [rows, words], a row sees the context in front of its sequence's rows and
    those of them whose bits are set in its words (``tree_masks``); a window has to be max_rows at least then."""
    if stream is not None or cache.index != _current_device():
        used = (*cache.tensors, *batch.tensors, q, out, workspace)
        return _on(cache.device, stream, used if tree is None else (*used, tree),
                   lambda: attend(cache, batch, q, scale, window, causal, out, want_lse, workspace, tree=tree))
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
    if tree is not None:
        _on_gpu(tree, "tree", torch.int64)
        if tree.device != device or tree.dim() != 2 or tree.shape[0] != n or not tree.is_contiguous():
            raise ValueError("tree must be contiguous [rows, words] on the cache's device")
        if not causal:
            raise ValueError("a tree says what each row sees: causal stays True")
    lse = torch.empty((n, heads), dtype=torch.float32, device=device) if want_lse else None
    a = T.tent_kv_attend_args(q.data_ptr(), out.data_ptr(), lse.data_ptr() if want_lse else None, q_stride, out_stride, None, 0, heads, window,
                              0 if causal else T.TENT_KV_ATTEND_ALL, 1.0 / math.sqrt(D) if scale is None else scale)
    L, need, ref = T.lib(), C.c_uint64(), C.byref(a)
    if tree is None:
        _check(L.tent_kv_attend_workspace(cache.ref, batch.ref, ref, C.byref(need)), "tent_kv_attend_workspace")
    else:
        _check(L.tent_kv_attend_tree_workspace(cache.ref, batch.ref, ref, C.byref(need)), "tent_kv_attend_tree_workspace")
    if need.value:
        if workspace is None:
            workspace = torch.empty(need.value, dtype=torch.uint8, device=device)
        elif not _on_gpu(workspace, "workspace", torch.uint8).is_contiguous() or workspace.device != device:
            raise ValueError("workspace must be contiguous, on the cache's device")
        a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel()
    if tree is None:
        _check(L.tent_kv_attend(cache.ref, batch.ref, ref, _stream(cache.index)), "tent_kv_attend")
    else:
        masks = T.tent_kv_tree(tree.data_ptr(), tree.shape[1], 0)
        _check(L.tent_kv_attend_tree(cache.ref, batch.ref, ref, C.byref(masks), _stream(cache.index)), "tent_kv_attend_tree")
    return (out, lse) if want_lse else out


def attend_workspace(cache: Cache, batch: Batch, q_heads: int, window: int = 0, causal: bool = True, tree: bool = False) -> int:
    """Bytes of workspace that attend takes for such a batch, with or without `tree`."""
    _together(cache, batch)
    bytes_of = T.tent_kv_attend_tree_workspace if tree else T.tent_kv_attend_workspace
    return bytes_of(cache.c, batch.c, T.tent_kv_attend_args(q_heads=q_heads, window=window, scale=1.0, flags=0 if causal else T.TENT_KV_ATTEND_ALL))


_PROBABILITIES = {**_TYPES, torch.float32: T.TENT_FP32}


def _vector(tensor, name, dtype, n, device):
    """A contiguous tensor of `n` values on `device`; its address."""
    if type(tensor) is torch.Tensor and tensor.dtype is dtype and tensor.shape == (n,) and tensor.device == device and not tensor.requires_grad and tensor.is_contiguous():
        return tensor.data_ptr()
    if not _on_gpu(tensor, name, dtype, (n,)).is_contiguous() or tensor.device != device:
        raise ValueError(f"{name} must be contiguous, on the batch's device")
    return tensor.data_ptr()


def _by_list(tensor, name, dtype, n_seqs, width, device):
    """A tensor [sequences, values] or [sequences, heads, values] of `width` values at least, lists at one distance; heads, distance."""
    if type(tensor) is torch.Tensor and tensor.dtype is dtype and tensor.device == device and not tensor.requires_grad and tensor.is_contiguous():
        shape = tensor.shape
        if len(shape) in (2, 3) and shape[0] == n_seqs and shape[-1] >= max(width, 1):
            return shape[1] if len(shape) == 3 else 1, shape[-1]
    _on_gpu(tensor, name, dtype)
    if tensor.device != device or tensor.dim() not in (2, 3) or tensor.shape[0] != n_seqs or tensor.shape[-1] < width:
        raise ValueError(f"{name} must be [sequences, (heads,) values] with {width} values at least, on the batch's device, not {tuple(tensor.shape)}")
    lists, stride = tensor.shape[1] if tensor.dim() == 3 else 1, tensor.stride()
    apart = stride[1] if tensor.dim() == 3 and lists > 1 else stride[0] if n_seqs > 1 else tensor.shape[-1]
    if (tensor.shape[-1] > 1 and stride[-1] != 1) or (n_seqs > 1 and stride[0] != lists * apart) or apart < tensor.shape[-1]:
        raise ValueError(f"{name} must have lists of contiguous values, all as far apart (strides {stride})")
    return lists, apart


def _meets(out, x):
    """Whether the bytes of `out`, which is contiguous, have any of `x`, whose rows are contiguous and all as far apart."""
    size, a = x.element_size(), out.data_ptr() - x.data_ptr()
    width = x.shape[-1] * size
    if not x.numel() or not out.numel():
        return False
    apart = min([stride for stride, n in zip(x.stride()[:-1], x.shape[:-1]) if n > 1], default=x.shape[-1]) * size
    first = max(0, (a - width) // apart + 1)                             # the first row that ends behind where `out` begins
    return first < x.numel() // x.shape[-1] and first * apart < a + out.numel() * out.element_size()


def _apart(out, name, used):
    """Refuses an output that other workgroups would still be reading as one of the tensors `used`."""
    for x in used:
        if x is not None and _meets(out, x):
            raise ValueError(f"{name} must not share memory with what the call reads")


def _like(tensor, lists, apart, known):
    """A new tensor laid out as one that _by_list has seen, with its values from place `known` of a list on."""
    shape = (tensor.shape[0], apart) if tensor.dim() == 2 else (tensor.shape[0], lists, apart)
    out = torch.empty(shape, dtype=tensor.dtype, device=tensor.device)
    if apart > tensor.shape[-1]:
        out = out[..., :tensor.shape[-1]]
    if tensor.shape[-1] > known:
        out[..., known:] = tensor[..., known:]
    return out


def verify(batch: Batch, target, tokens, accept, next, parents=None, draft=None, path=None, workspace=None, stream=None):
    """Which of the batch's rows stand, and what comes behind them: path [sequences, max_rows] (int32, rows of the sequence, the first of
    them first, then -1), counts [sequences] and token [sequences].

    target: [rows, vocab], probabilities of the token behind each row, float32, bfloat16 or float16.  tokens: int32 [rows], drafted
    tokens, of which the first of a sequence stands for the one that is decided already.  parents: int32 [rows], the row of its
    sequence that a row is behind; the one before unless given.  draft: as target, the probabilities that the rows behind a row
    were drawn from, each by itself; None: they were chosen without drawing.  accept: float32 [rows] and next: float32 [sequences],
    random numbers, 0 <= u < 1.  path: int32 [sequences, max_rows] to use instead of a new one, apart from the tensors that are read.
    workspace: a contiguous uint8 tensor of at least verify_workspace bytes, likewise."""
    if stream is not None or batch.device.index != _current_device():
        used = [x for x in (*batch.tensors, target, tokens, accept, next, parents, draft, path, workspace) if x is not None]
        return _on(batch.device, stream, used, lambda: verify(batch, target, tokens, accept, next, parents, draft, path, workspace))
    n, n_seqs, most, device = batch.n_rows, batch.c.n_seqs, batch.c.max_rows, batch.device
    if not isinstance(target, torch.Tensor) or target.dim() != 2 or target.dtype not in _PROBABILITIES:
        raise ValueError("target must be float32, bfloat16 or float16 [rows, vocab]")
    vocab, strides = target.shape[1], [0, 0]
    for i, (x, name) in enumerate(((target, "target"), (draft, "draft"))):
        if x is None:
            continue
        if type(x) is not torch.Tensor or x.dtype is not target.dtype or x.shape != (n, vocab) or x.device != device or x.requires_grad:
            _on_gpu(x, name, target.dtype, (n, vocab))
            if x.device != device:
                raise ValueError(f"{name} must be on the batch's device")
        stride = x.stride()
        if (vocab > 1 and stride[1] != 1) or (n > 1 and stride[0] < vocab):
            raise ValueError(f"{name} must have contiguous rows (strides {stride})")
        strides[i] = stride[0] if n > 1 else vocab
    a = T.tent_kv_verify_args(target.data_ptr(), draft.data_ptr() if draft is not None else None, *strides, _vector(tokens, "tokens", torch.int32, n, device),
                              _vector(parents, "parents", torch.int32, n, device) if parents is not None else None,
                              _vector(accept, "accept", torch.float32, n, device), _vector(next, "next", torch.float32, n_seqs, device))
    if path is None:
        path = torch.empty((n_seqs, most), dtype=torch.int32, device=device)
    elif not _on_gpu(path, "path", torch.int32, (n_seqs, most)).is_contiguous() or path.device != device:
        raise ValueError("path must be contiguous, on the batch's device")
    else:
        _apart(path, "path", (*batch.tensors, target, tokens, accept, next, parents, draft))
    counts, token = torch.empty((n_seqs,), dtype=torch.int32, device=device), torch.empty((n_seqs,), dtype=torch.int32, device=device)
    a.path, a.counts, a.token = path.data_ptr(), counts.data_ptr(), token.data_ptr()
    a.vocab, a.path_stride, a.type = vocab, most, _PROBABILITIES[target.dtype]
    L, need, ref = T.lib(), C.c_uint64(), C.byref(a)
    _check(L.tent_kv_verify_workspace(batch.ref, ref, C.byref(need)), "tent_kv_verify_workspace")
    if need.value:
        if workspace is None:
            workspace = torch.empty(need.value, dtype=torch.uint8, device=device)
        elif not _on_gpu(workspace, "workspace", torch.uint8).is_contiguous() or workspace.device != device:
            raise ValueError("workspace must be contiguous, on the batch's device")
        a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel()
    _check(L.tent_kv_verify(batch.ref, ref, _stream(device.index)), "tent_kv_verify")
    return path, counts, token


def verify_workspace(batch: Batch, vocab: int, parents: bool = False, draft: bool = False) -> int:
    """Bytes of workspace that verify takes for such a batch, with or without `parents` and `draft`."""
    return T.tent_kv_verify_workspace(batch.c, T.tent_kv_verify_args(vocab=vocab, parents=4 if parents else None, draft=4 if draft else None, type=T.TENT_FP32))


def weigh(cache: Cache, batch: Batch, q, lse, weights=None, per_head: bool = True, scale: float = None, window: int = 0, causal: bool = True, out=None,
          workspace=None, stream=None):
    """`weights` and what the batch's rows add to them: the attention weight that each token gets from the rows that see it, [sequences,
    kv_heads, max_kv] (float32; summed over the query heads of a head) or, without per_head, [sequences, max_kv] summed over all heads.

    q, scale, window, causal: as attend had them (without `tree`: of a tree the rows that stand can be weighed, once keep has made them the
    sequence); lse: float32 [rows, q_heads], what it has said with want_lse.  weights: None for zeros; its lists may be longer than max_kv.  out may be weights.  workspace: a contiguous uint8 tensor of at least weigh_workspace bytes
    to use instead of a new one."""
    if stream is not None or cache.index != _current_device():
        used = [x for x in (*cache.tensors, *batch.tensors, q, lse, weights, out, workspace) if x is not None]
        return _on(cache.device, stream, used, lambda: weigh(cache, batch, q, lse, weights, per_head, scale, window, causal, out, workspace))
    _together(cache, batch)
    n, n_seqs, D, device = batch.n_rows, batch.c.n_seqs, cache.head_dim, cache.device
    heads = q.shape[1] if isinstance(q, torch.Tensor) and q.dim() == 3 else 0
    q_stride = _rows(q, "q", cache.dtype, n, heads, D, device)
    if not _on_gpu(lse, "lse", torch.float32, (n, heads)).is_contiguous() or lse.device != device:
        raise ValueError("lse must be contiguous, on the cache's device")
    if not 0 <= window < 1 << 31:
        raise ValueError("window must be 0 or more and below 2^31")
    lists = cache.kv_heads if per_head else 1
    given = _by_list(weights, "weights", torch.float32, n_seqs, batch.max_kv, device) if weights is not None else None
    if out is None:
        out = torch.empty((n_seqs, lists, batch.max_kv) if per_head else (n_seqs, batch.max_kv), dtype=torch.float32, device=device) if given is None \
            else _like(weights, *given, batch.max_kv)
    made = _by_list(out, "out", torch.float32, n_seqs, batch.max_kv, device)
    if made[0] != lists or given not in (None, made):
        raise ValueError("weights and out must have a list for each head (or, without per_head, one), and the same strides")
    a = T.tent_kv_weigh_args(q.data_ptr(), lse.data_ptr(), weights.data_ptr() if weights is not None else None, out.data_ptr(), q_stride, made[1], None, 0,
                             heads, lists, window, 0 if causal else T.TENT_KV_ATTEND_ALL, 1.0 / math.sqrt(D) if scale is None else scale, 0)
    L, ref = T.lib(), C.byref(a)
    if lists != cache.kv_heads:                                          # with a list for each head none is needed
        need = C.c_uint64()
        _check(L.tent_kv_weigh_workspace(cache.ref, batch.ref, ref, C.byref(need)), "tent_kv_weigh_workspace")
        if need.value:
            if workspace is None:
                workspace = torch.empty(need.value, dtype=torch.uint8, device=device)
            elif not _on_gpu(workspace, "workspace", torch.uint8).is_contiguous() or workspace.device != device:
                raise ValueError("workspace must be contiguous, on the cache's device")
            a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel()
    _check(L.tent_kv_weigh(cache.ref, batch.ref, ref, _stream(cache.index)), "tent_kv_weigh")
    return out


def weigh_workspace(cache: Cache, batch: Batch, q_heads: int, per_head: bool = True) -> int:
    """Bytes of workspace that weigh takes for such a batch."""
    _together(cache, batch)
    return T.tent_kv_weigh_workspace(cache.c, batch.c, T.tent_kv_weigh_args(q_heads=q_heads, n_lists=cache.kv_heads if per_head else 1, scale=1.0))


def choose(batch: Batch, weights, budget: int, first: int = 0, recent: int = 0, workspace=None, stream=None):
    """Which tokens every sequence of the batch keeps: lists [sequences, (heads,) budget] (int32, ascending, then -1) and counts [sequences].
    All where there are no more than `budget`; else the `first` first, the `recent` last and those of the greatest weights.
    weights: float32 [sequences, (heads,) max_kv or more], as weigh makes them.  workspace: a contiguous uint8 tensor of at least
    choose_workspace bytes to use instead of a new one."""
    if stream is not None or batch.device.index != _current_device():
        used = (*batch.tensors, weights) if workspace is None else (*batch.tensors, weights, workspace)
        return _on(batch.device, stream, used, lambda: choose(batch, weights, budget, first, recent, workspace))
    n_seqs, device = batch.c.n_seqs, batch.device
    lists, apart = _by_list(weights, "weights", torch.float32, n_seqs, batch.max_kv, device)
    if not 1 <= budget <= 1 << 30 or first < 0 or recent < 0 or first + recent > budget:
        raise ValueError("budget must be 1 or more, and hold the first and the recent tokens")
    out = torch.empty((*weights.shape[:-1], budget), dtype=torch.int32, device=device)
    counts = torch.empty((n_seqs,), dtype=torch.int32, device=device)
    a = T.tent_kv_choose_args(weights.data_ptr(), out.data_ptr(), counts.data_ptr(), apart, budget, None, 0, lists, budget, first, recent)
    L, ref = T.lib(), C.byref(a)
    if batch.max_kv > T.TENT_KV_CHOOSE_WHOLE:                            # up to there none is needed
        need = C.c_uint64()
        _check(L.tent_kv_choose_workspace(batch.ref, ref, C.byref(need)), "tent_kv_choose_workspace")
        if need.value:
            if workspace is None:
                workspace = torch.empty(need.value, dtype=torch.uint8, device=device)
            elif not _on_gpu(workspace, "workspace", torch.uint8).is_contiguous() or workspace.device != device:
                raise ValueError("workspace must be contiguous, on the batch's device")
            a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel()
    _check(L.tent_kv_choose(batch.ref, ref, _stream(device.index)), "tent_kv_choose")
    return out, counts


def choose_workspace(batch: Batch, lists: int = 1) -> int:
    """Bytes of workspace that choose takes for such a batch and so many lists of each sequence."""
    return T.tent_kv_choose_workspace(batch.c, T.tent_kv_choose_args(n_lists=lists))


def keep(cache: Cache, batch: Batch, lists, counts, rows: bool = False, to_table=None, weights=None, weights_out=None, kv_len_out=None, stream=None):
    """Move the tokens that every sequence keeps together; their number afterwards (int32 [sequences], a new tensor unless given), and with
    `weights` these moved along.

    Token j becomes what token lists[sequence, (head,) j] was, for j below counts[sequence]; one list for all heads or one for each.  With
    rows=True lists name rows of the sequence (verify's path) and the context in front of them stays.  In place, unless to_table
    (int32 [sequences, pages]) names other pages to write to.  weights: float32 [sequences, (heads,) max_kv or more], moved to weights_out
    (in place itself unless given; a new tensor with to_table), behind the last kept token 0.  Keys keep the rotations that they have:
    after an eviction append takes `positions` that go on from the tokens' own, not from the shorter length.  kv_len_out shares no memory with what is
    read, nor with the batch's kv_len: heads whose turn comes later still read that."""
    if stream is not None or cache.index != _current_device():
        used = [x for x in (*cache.tensors, *batch.tensors, lists, counts, to_table, weights, weights_out, kv_len_out) if x is not None]
        return _on(cache.device, stream, used, lambda: keep(cache, batch, lists, counts, rows, to_table, weights, weights_out, kv_len_out))
    _together(cache, batch)
    n_seqs, device = batch.c.n_seqs, cache.device
    n_lists, apart = _by_list(lists, "lists", torch.int32, n_seqs, 0, device)
    if n_lists not in (1, cache.kv_heads):
        raise ValueError("lists must be one for every head of the cache, or one for all")
    a = T.tent_kv_keep_args(lists.data_ptr(), _vector(counts, "counts", torch.int32, n_seqs, device))
    if to_table is not None:
        _on_gpu(to_table, "to_table", torch.int32)
        if to_table.dim() != 2 or to_table.shape[0] != n_seqs or to_table.device != device or (to_table.shape[1] > 1 and to_table.stride(1) != 1):
            raise ValueError("to_table must be [sequences, pages] with contiguous rows, on the cache's device")
        entries = to_table.shape[1]
        to_stride = to_table.stride(0) if n_seqs > 1 else entries
        if n_seqs and not entries:                                       # no address either: it would be taken for none
            raise ValueError("to_table names no pages")
        if not entries <= to_stride < 1 << 32:
            raise ValueError("rows of to_table overlap, or are too far apart")
        a.to_table, a.to_stride, a.to_entries = to_table.data_ptr(), to_stride, entries
    if weights is not None:
        a.n_weights, a.weights_stride = _by_list(weights, "weights", torch.float32, n_seqs, batch.max_kv, device)
        if weights_out is None:
            weights_out = weights if to_table is None else _like(weights, a.n_weights, a.weights_stride, batch.max_kv)
        if _by_list(weights_out, "weights_out", torch.float32, n_seqs, batch.max_kv, device) != (a.n_weights, a.weights_stride):
            raise ValueError("weights and weights_out must have the same heads and strides")
        if a.n_weights not in (n_lists, cache.kv_heads):
            raise ValueError("weights must have as many heads as lists, or one list for all heads")
        a.weights, a.weights_out = weights.data_ptr(), weights_out.data_ptr()
    elif weights_out is not None:
        raise ValueError("weights_out goes with weights")
    if kv_len_out is None:
        kv_len_out = torch.empty((n_seqs,), dtype=torch.int32, device=device)
        a.kv_len_out = kv_len_out.data_ptr()
    else:
        a.kv_len_out = _vector(kv_len_out, "kv_len_out", torch.int32, n_seqs, device)
        _apart(kv_len_out, "kv_len_out", (batch.page_table, batch.errors, lists, to_table, weights))
    a.list_stride, a.n_lists, a.most, a.flags = apart, n_lists, lists.shape[-1], T.TENT_KV_KEEP_ROWS if rows else 0
    _check(T.lib().tent_kv_keep(cache.ref, batch.ref, C.byref(a), _stream(cache.index)), "tent_kv_keep")
    return kv_len_out if weights is None else (kv_len_out, weights_out)
