"""Paged pools: block tables, slot maps, cache writes and tree attention.

A pool of equal pages holds the keys and values of the sequences that a model
is answering.  Its pages' kinds are the same uint8 array that window_search and
first_fit read, so they work on it too.  As in the rest of the package, every
step runs in the HIP kernels of libcoop.so, calls are asynchronous on torch's
current stream (or the `stream` argument), and each operator comes as a
prepared call (a class whose `launch` can be repeated or captured into a graph)
and as a function.  A function called with `stream` runs behind what is queued
on the current stream; its inputs may be dropped at once, its results are there
when `stream` is done.

Caches are tensors [pages, page_size, heads, dim] of bfloat16, float16 or
float8_e4m3fn, in any order of the first three dimensions in memory (a
transposed view, or one half of a tensor that holds keys and values together).

The operators serve a model that answers and have no gradients: while torch
records them, tensors that require them are refused, and so are those that carry
tangents.
"""
from __future__ import annotations

import ctypes
import functools
from typing import Optional

import torch
from torch.autograd import forward_ad

from . import COOP_EVICTABLE, COOP_PINNED, _check, _ptr, load_library

# (torch without GPU support lacks these)
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None)

_TYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float8_e4m3fn: 2}


class CoopCache(ctypes.Structure):
    """coop_cache_t."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("k_stride", ctypes.c_uint64 * 3), ("v_stride", ctypes.c_uint64 * 3),
                ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("num_pages", ctypes.c_uint64), ("page_size", ctypes.c_uint64),
                ("heads", ctypes.c_uint64), ("dim", ctypes.c_uint64), ("type", ctypes.c_int32)]


class CoopRows(ctypes.Structure):
    """coop_rows_t."""
    _fields_ = [("data", ctypes.c_void_p), ("stride", ctypes.c_uint64 * 2)]


@functools.lru_cache(maxsize=64)
def _stream(handle: int, device):
    # (ExternalStream takes 0 for no stream and makes one)
    return torch.cuda.ExternalStream(handle, device) if handle else torch.cuda.default_stream(device)


def _gpu(device):
    if device.type != "cuda":
        raise ValueError(f"paged pools are worked on by the GPU; tensors are on {device} "
                         "(there is no CPU fallback)")
    return device


def _no_gradients(k, v, k_cache, v_cache, k_scale, v_scale, q=None, out=None) -> None:
    """Refuses tensors whose gradients or tangents would be lost."""
    recorded = torch.is_grad_enabled() and (
        k.requires_grad or v.requires_grad or k_cache.requires_grad or v_cache.requires_grad
        or k_scale is not None and k_scale.requires_grad
        or v_scale is not None and v_scale.requires_grad
        or q is not None and q.requires_grad or out is not None and out.requires_grad)
    # (tensors carry tangents only inside of a level; -1: there is none)
    if not recorded and getattr(forward_ad, "_current_level", 0) < 0:
        return
    for name, t in dict(k=k, v=v, k_cache=k_cache, v_cache=v_cache, k_scale=k_scale,
                        v_scale=v_scale, q=q, out=out).items():
        if t is None:
            continue
        if recorded and t.requires_grad:
            raise ValueError(f"{name} requires gradients, which paged pools do not have (detach it, "
                             "or call under torch.no_grad())")
        if forward_ad.unpack_dual(t).tangent is not None:
            raise ValueError(f"{name} carries a tangent, which paged pools do not pass on")


def _vector(t: torch.Tensor, name: str, dtype, device, *shape) -> torch.Tensor:
    if t.dtype != dtype and not (dtype == torch.int64 and t.dtype == torch.uint64):
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {shape}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _strides(t: torch.Tensor, name: str, elements: int):
    """The strides of the leading dimensions (0 for one of size 1)."""
    stride = t.stride()
    if stride[-1] != 1 and t.shape[-1] != 1:
        raise ValueError(f"{name}'s last dimension must be contiguous")
    bad = t.data_ptr() % 16
    for x in stride[:-1]:
        bad |= x % elements
    if bad:  # (unless the offending dimension is one that is never stepped along)
        stride = tuple(0 if n == 1 else x for n, x in zip(t.shape, stride))
        if t.data_ptr() % 16 or any(x % elements for x in stride[:-1]):
            raise ValueError(f"{name}'s rows must start at multiples of 16 bytes")
    return stride[:-1]


def _rows(t: torch.Tensor, name: str, dtype, device, shape) -> CoopRows:
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {shape}, got {tuple(t.shape)}")
    if shape[0] == 0:
        return CoopRows(None, (0, 0))
    return CoopRows(t.data_ptr(), _strides(t, name, 8))


def _cache(k_cache, v_cache, k_scale, v_scale, dtype, device) -> CoopCache:
    shape, kind = k_cache.shape, k_cache.dtype
    if len(shape) != 4 or shape != v_cache.shape:
        raise ValueError("k_cache and v_cache must have one shape [pages, page_size, heads, dim], "
                         f"got {tuple(shape)} and {tuple(v_cache.shape)}")
    if v_cache.dtype != kind or kind not in (dtype, torch.float8_e4m3fn):
        raise TypeError(f"k_cache and v_cache must both be {dtype} or torch.float8_e4m3fn, got "
                        f"{kind} and {v_cache.dtype}")
    if k_cache.device != device or v_cache.device != device:
        raise ValueError(f"the cache is on {k_cache.device} and {v_cache.device}, expected {device}")
    pages, page_size, heads, dim = shape
    elements, ks, vs = 8, None, None
    if kind == torch.float8_e4m3fn:
        elements = 16
        if k_scale is None or v_scale is None:
            raise ValueError("a float8_e4m3fn cache needs k_scale and v_scale")
        ks = _vector(k_scale, "k_scale", torch.float32, device, heads).data_ptr()
        vs = _vector(v_scale, "v_scale", torch.float32, device, heads).data_ptr()
    elif k_scale is not None or v_scale is not None:
        raise ValueError(f"a {kind} cache has no k_scale or v_scale")
    if k_cache.numel() == 0:
        return CoopCache(None, None, (0, 0, 0), (0, 0, 0), ks, vs, pages, page_size, heads, dim,
                         _TYPES[kind])
    return CoopCache(k_cache.data_ptr(), v_cache.data_ptr(), _strides(k_cache, "k_cache", elements),
                     _strides(v_cache, "v_cache", elements), ks, vs, pages, page_size, heads, dim,
                     _TYPES[kind])


def _workspace(workspace: Optional[torch.Tensor], need: int, device):
    """(the workspace to keep alive, its address, its bytes)."""
    if workspace is None:
        if need == 0:
            return None, None, 0
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
        return workspace, workspace.data_ptr(), need
    if workspace.device != device or not workspace.is_contiguous():
        raise ValueError(f"workspace must be contiguous memory on {device}")
    held = workspace.numel() * workspace.element_size()
    if held < need:
        raise ValueError(f"workspace holds {held} bytes, needs {need}")
    return workspace, workspace.data_ptr(), held


def _capturing(stream) -> bool:
    with torch.cuda.stream(stream):
        return torch.cuda.is_current_stream_capturing()


class _Call:
    """A prepared call: the C function, its arguments (all but the stream) and
    the tensors that it uses (None where there is none), which it keeps alive."""

    _met = ()  # the other streams that the call was launched on

    def _prepare(self, device, fn, args, tensors):
        self.device, self._fn, self._args, self._tensors = device, fn, args, tensors
        self._home = _current_stream(device.index)

    def _meet(self, stream: int) -> None:
        """Puts `stream` behind what is queued on the stream that the call was
        made on, where the memory that it allocated may still be in use from
        before, and keeps all of its tensors' memory (inputs may be dropped as
        soon as the call is) from being handed out again before `stream` is
        done."""
        other = _stream(stream, self.device)
        home = _stream(self._home, self.device)
        if _capturing(other) or torch.cuda.is_current_stream_capturing():
            # a graph cannot wait for what is outside of it, and its owner keeps the call
            # (the default stream, 0, is never captured)
            if not (self._home and _capturing(home)):
                return
            other.wait_stream(home)
        elif not home.query():  # (asking is far cheaper than waiting for what is done)
            other.wait_stream(home)
        for t in self._tensors:
            if t is not None:
                t.record_stream(other)
        self._met += (stream,)

    def launch(self, stream: Optional[int] = None) -> None:
        """Enqueues the call on `stream` (default: torch's current stream of
        the tensors' device).  The first launch on another stream than the one
        that was current when the call was made waits for what is queued there
        by then; apart from that, the inputs are to be ready on `stream`, and
        launches, which share results and workspace, in order.  A call that a
        graph captured is to be kept as long as the graph."""
        index = self.device.index
        if stream is None:
            stream = _current_stream(index)
        if stream != self._home and stream not in self._met:
            self._meet(stream)
        if _current_device() == index:
            status = self._fn(*self._args, stream)
        else:
            with torch.cuda.device(self.device):
                status = self._fn(*self._args, stream)
        if status:
            _check(status)


@functools.lru_cache(maxsize=1024)
def page_tables_workspace_size(num_pages: int, num_requests: int) -> int:
    """Device workspace bytes coop_page_tables needs."""
    out = ctypes.c_size_t(0)
    _check(load_library().coop_page_tables_workspace_size(int(num_pages), int(num_requests),
                                                          ctypes.byref(out)))
    return out.value


class PageTables(_Call):
    """A prepared coop_page_tables call: brings the block tables of a batch of
    sequences in line with their new lengths.

    kind: uint8 [pages] (0 free, 1 evictable, 2 pinned); table: int32
    [requests, columns], page numbers; held: int32 [requests], the entries in
    use of each row; lengths: int64 [requests], the tokens that each sequence is
    to hold.  Rows that hold more pages than ceil(length / page_size) give their
    last ones back; then rows that need more take the lowest free pages, in the
    rows' order, which become `taken`.  Once a row cannot have all that it
    needs, it and every later one that needs more keep what they had.  A page
    that a row names must not be set free in `kind` by hand: what is to be
    evicted leaves its row by a shorter length.

    Results: `table`, `held`, `kind` (new tensors; with out=(table, held, kind)
    written there, and these may be the inputs themselves), `status` (int32
    [1]: bit 0, a row was refused for want of free pages; bit 1, one needs more
    than a row has columns) and `free` (int64 [1], free pages left)."""

    def __init__(self, kind, table, held, lengths, page_size: int, *, taken: int = COOP_PINNED,
                 out=None, workspace: Optional[torch.Tensor] = None):
        device = _gpu(kind.device)
        if kind.dim() != 1 or table.dim() != 2:
            raise ValueError("kind must have shape [pages] and table [requests, columns], got "
                             f"{tuple(kind.shape)} and {tuple(table.shape)}")
        pages, (rows, cols) = kind.numel(), table.shape
        _vector(kind, "kind", torch.uint8, device, pages)
        _vector(table, "table", torch.int32, device, rows, cols)
        _vector(held, "held", torch.int32, device, rows)
        _vector(lengths, "lengths", torch.int64, device, rows)
        if page_size < 1:
            raise ValueError(f"page_size must be at least 1, got {page_size}")
        if taken not in (COOP_EVICTABLE, COOP_PINNED):
            raise ValueError(f"taken must be COOP_EVICTABLE or COOP_PINNED, got {taken}")
        if out is None:
            out = (torch.empty_like(table), torch.empty_like(held), torch.empty_like(kind))
        else:
            _vector(out[0], "out[0]", torch.int32, device, rows, cols)
            _vector(out[1], "out[1]", torch.int32, device, rows)
            _vector(out[2], "out[2]", torch.uint8, device, pages)
        self.table, self.held, self.kind = out
        self.status = torch.empty(1, dtype=torch.int32, device=device)
        self.free = torch.empty(1, dtype=torch.int64, device=device)
        self.workspace, ws, ws_bytes = _workspace(
            workspace, page_tables_workspace_size(pages, rows), device)
        self._prepare(device, load_library().coop_page_tables,
                      (_ptr(kind), pages, _ptr(table), rows, cols, _ptr(held), _ptr(lengths),
                       page_size, taken, _ptr(self.table), _ptr(self.held), _ptr(self.kind),
                       self.status.data_ptr(), self.free.data_ptr(), ws, ws_bytes),
                      (kind, table, held, lengths, self.table, self.held, self.kind, self.status,
                       self.free, self.workspace))

    def __call__(self, stream: Optional[int] = None):
        self.launch(stream)
        return self.table, self.held, self.kind, self.status, self.free


def page_tables(kind, table, held, lengths, page_size: int, *, taken: int = COOP_PINNED, out=None,
                workspace: Optional[torch.Tensor] = None, stream: Optional[int] = None):
    """One PageTables call; returns (table, held, kind, status, free)."""
    return PageTables(kind, table, held, lengths, page_size, taken=taken, out=out,
                      workspace=workspace)(stream)


class SlotMap(_Call):
    """A prepared coop_slot_map call: the slot (page * page_size + place) of
    each of num_tokens new tokens.  token_offsets: int64 [requests + 1];
    sequence b's new tokens are the last token_offsets[b+1] - token_offsets[b]
    of its lengths[b].  -1 where a token has no place.  Result: `slots`, int64
    [num_tokens]."""

    def __init__(self, table, held, lengths, token_offsets, num_tokens: int, page_size: int,
                 num_pages: int, out: Optional[torch.Tensor] = None):
        device = _gpu(table.device)
        if table.dim() != 2:
            raise ValueError(f"table must have shape [requests, columns], got {tuple(table.shape)}")
        rows, cols = table.shape
        _vector(table, "table", torch.int32, device, rows, cols)
        _vector(held, "held", torch.int32, device, rows)
        _vector(lengths, "lengths", torch.int64, device, rows)
        _vector(token_offsets, "token_offsets", torch.int64, device, rows + 1)
        if num_tokens < 0 or page_size < 1 or num_pages < 0:
            raise ValueError(f"num_tokens {num_tokens}, page_size {page_size} and num_pages "
                             f"{num_pages} must be at least 0, 1 and 0")
        if out is None:
            out = torch.empty(num_tokens, dtype=torch.int64, device=device)
        self.slots = _vector(out, "out", torch.int64, device, num_tokens)
        self._prepare(device, load_library().coop_slot_map,
                      (_ptr(table), rows, cols, _ptr(held), _ptr(lengths),
                       token_offsets.data_ptr(), num_tokens, page_size, num_pages,
                       _ptr(self.slots)), (table, held, lengths, token_offsets, self.slots))

    def __call__(self, stream: Optional[int] = None) -> torch.Tensor:
        self.launch(stream)
        return self.slots


def slot_map(table, held, lengths, token_offsets, num_tokens: int, page_size: int, num_pages: int,
             *, out: Optional[torch.Tensor] = None, stream: Optional[int] = None) -> torch.Tensor:
    """One SlotMap call; returns int64 [num_tokens]."""
    return SlotMap(table, held, lengths, token_offsets, num_tokens, page_size, num_pages,
                   out)(stream)


class CacheWrite(_Call):
    """A prepared coop_cache_write call: rows of keys and values ([tokens,
    heads, dim], bfloat16 or float16) to their slots of the pool (int64
    [tokens]; tokens without a slot in the pool are skipped, and slots must
    differ).  A float8_e4m3fn cache stores them divided by their head's scale
    (float32 [heads]), limited to +-448."""

    def __init__(self, k, v, slots, k_cache, v_cache, *, k_scale=None, v_scale=None):
        device = _gpu(k.device)
        if k.dtype not in (torch.bfloat16, torch.float16):
            raise TypeError(f"k must be torch.bfloat16 or torch.float16, got {k.dtype}")
        if k.dim() != 3:
            raise ValueError(f"k must have shape [tokens, heads, dim], got {tuple(k.shape)}")
        _no_gradients(k, v, k_cache, v_cache, k_scale, v_scale)
        cache = _cache(k_cache, v_cache, k_scale, v_scale, k.dtype, device)
        shape = n, _, _ = (k.shape[0], cache.heads, cache.dim)
        k_rows = _rows(k, "k", k.dtype, device, shape)
        v_rows = _rows(v, "v", k.dtype, device, shape)
        _vector(slots, "slots", torch.int64, device, n)
        self.k_cache, self.v_cache = k_cache, v_cache
        self._prepare(device, load_library().coop_cache_write,
                      (ctypes.byref(k_rows), ctypes.byref(v_rows), _TYPES[k.dtype], _ptr(slots), n,
                       ctypes.byref(cache)), (k, v, slots, k_cache, v_cache, k_scale, v_scale))

    def __call__(self, stream: Optional[int] = None):
        self.launch(stream)
        return self.k_cache, self.v_cache


def cache_write(k, v, slots, k_cache, v_cache, *, k_scale=None, v_scale=None,
                stream: Optional[int] = None):
    """One CacheWrite call; returns (k_cache, v_cache), written in place."""
    return CacheWrite(k, v, slots, k_cache, v_cache, k_scale=k_scale, v_scale=v_scale)(stream)


@functools.lru_cache(maxsize=1024)
def tree_attention_workspace_size(num_requests: int, num_tokens: int, q_heads: int, heads: int,
                                  dim: int) -> int:
    """Device workspace bytes coop_tree_attention needs."""
    out = ctypes.c_size_t(0)
    _check(load_library().coop_tree_attention_workspace_size(
        int(num_requests), int(num_tokens), int(q_heads), int(heads), int(dim), ctypes.byref(out)))
    return out.value


class TreeAttention(_Call):
    """A prepared coop_tree_attention call: attention of new tokens over the
    cached tokens of their requests and over one another.

    q [tokens, q_heads, dim], k and v [tokens, heads, dim] (bfloat16 or
    float16): the new tokens; request b's are token_offsets[b] to
    token_offsets[b+1] (int64 [requests + 1]).  lengths (int64 [requests]): the
    tokens in the pool, on the pages of table's rows (int32 [requests,
    columns]).  parents (int32 [tokens]): the request-local number of each
    token's parent in its request's tree, -1 where it follows the cached tokens
    directly; a token sees the cached tokens, its ancestors and itself.
    parents=None: a chain, each token the parent of the next (a prompt or a
    piece of one; single tokens).  A parent that is neither -1 nor an earlier
    token makes its token void: a zero row, which no other token sees.
    scale: of the products, dim ** -0.5 by default.  Result: `out` [tokens,
    q_heads, dim] of q's type; rows past token_offsets[requests] (a padded
    batch) are not written."""

    def __init__(self, q, k, v, k_cache, v_cache, table, lengths, token_offsets, parents=None, *,
                 scale: Optional[float] = None, k_scale=None, v_scale=None,
                 out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
        device = _gpu(q.device)
        if q.dtype not in (torch.bfloat16, torch.float16):
            raise TypeError(f"q must be torch.bfloat16 or torch.float16, got {q.dtype}")
        if q.dim() != 3 or table.dim() != 2:
            raise ValueError("q must have shape [tokens, q_heads, dim] and table [requests, "
                             f"columns], got {tuple(q.shape)} and {tuple(table.shape)}")
        _no_gradients(k, v, k_cache, v_cache, k_scale, v_scale, q, out)
        cache = _cache(k_cache, v_cache, k_scale, v_scale, q.dtype, device)
        n, q_heads, dim = q.shape
        if cache.heads == 0 or q_heads == 0 or q_heads % cache.heads:
            raise ValueError(f"{q_heads} query heads cannot share {cache.heads} key/value heads")
        requests, cols = table.shape
        q_rows = _rows(q, "q", q.dtype, device, (n, q_heads, cache.dim))
        k_rows = _rows(k, "k", q.dtype, device, (n, cache.heads, cache.dim))
        v_rows = _rows(v, "v", q.dtype, device, (n, cache.heads, cache.dim))
        _vector(table, "table", torch.int32, device, requests, cols)
        _vector(lengths, "lengths", torch.int64, device, requests)
        _vector(token_offsets, "token_offsets", torch.int64, device, requests + 1)
        if parents is not None:
            _vector(parents, "parents", torch.int32, device, n)
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
        else:
            _vector(out, "out", q.dtype, device, n, q_heads, dim)
        self.out = out
        self.workspace, ws, ws_bytes = _workspace(
            workspace, tree_attention_workspace_size(requests, n, q_heads, cache.heads, dim),
            device)
        self._prepare(device, load_library().coop_tree_attention,
                      (ctypes.byref(q_rows), ctypes.byref(k_rows), ctypes.byref(v_rows),
                       _TYPES[q.dtype], q_heads, n, token_offsets.data_ptr(),
                       None if parents is None else _ptr(parents), ctypes.byref(cache), _ptr(table),
                       cols, _ptr(lengths), requests,
                       dim ** -0.5 if scale is None else float(scale), _ptr(out), ws, ws_bytes),
                      (q, k, v, k_cache, v_cache, table, lengths, token_offsets, parents, k_scale,
                       v_scale, out, self.workspace))

    def __call__(self, stream: Optional[int] = None) -> torch.Tensor:
        self.launch(stream)
        return self.out


def tree_attention(q, k, v, k_cache, v_cache, table, lengths, token_offsets, parents=None, *,
                   scale: Optional[float] = None, k_scale=None, v_scale=None,
                   out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                   stream: Optional[int] = None) -> torch.Tensor:
    """One TreeAttention call; returns [tokens, q_heads, dim]."""
    return TreeAttention(q, k, v, k_cache, v_cache, table, lengths, token_offsets, parents,
                         scale=scale, k_scale=k_scale, v_scale=v_scale, out=out,
                         workspace=workspace)(stream)


def _declare(lib) -> None:
    """The C signatures of the functions above."""
    u64, vp, sz, i32 = ctypes.c_uint64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32
    rows, cache, size_out = (ctypes.POINTER(CoopRows), ctypes.POINTER(CoopCache),
                             ctypes.POINTER(sz))
    lib.coop_page_tables_workspace_size.argtypes = [u64, u64, size_out]
    lib.coop_page_tables.argtypes = [vp, u64, vp, u64, u64, vp, vp, u64, ctypes.c_uint8, vp, vp,
                                     vp, vp, vp, vp, sz, vp]
    lib.coop_slot_map.argtypes = [vp, u64, u64, vp, vp, vp, u64, u64, u64, vp, vp]
    lib.coop_cache_write.argtypes = [rows, rows, i32, vp, u64, cache, vp]
    lib.coop_tree_attention_workspace_size.argtypes = [u64, u64, u64, u64, u64, size_out]
    lib.coop_tree_attention.argtypes = [rows, rows, rows, i32, u64, u64, vp, vp, cache, vp, u64,
                                        vp, u64, ctypes.c_float, vp, vp, sz, vp]
    for name in ("coop_page_tables_workspace_size", "coop_page_tables", "coop_slot_map",
                 "coop_cache_write", "coop_tree_attention_workspace_size", "coop_tree_attention"):
        getattr(lib, name).restype = ctypes.c_int
