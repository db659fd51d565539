"""Thin ctypes binding of the paged key-value cache's C ABI (include/ic_kv.h).

Argument checks and marshalling only: every step runs in the CUDA library, torch provides device
memory and streams.  `ICPagedKV` owns a handle together with its tensors.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional

import torch

from . import binding
from .binding import IC_ERR_INVALID, IC_OK, ICCacheError, ic_cache_last_error

IC_KV_BF16, IC_KV_F16 = 0, 1
IC_KV_MAX_HEAD_DIM, IC_KV_MAX_PAGE, IC_KV_MAX_SEQS = 256, 256, 16384


class ic_kv_opts_t(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32)] + [(n, ctypes.c_int32) for n in (
        "device", "dtype", "n_pages", "n_layers", "n_kv_heads", "page_size", "head_dim", "max_seqs", "max_pages")] + [
        (n, ctypes.c_void_p) for n in ("pool", "tables", "lengths", "refs", "stream", "workspace")] + [
        ("workspace_bytes", ctypes.c_size_t)]


class ic_kv_attend_t(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("layer", ctypes.c_int32), ("n", ctypes.c_int32), ("n_heads", ctypes.c_int32),
                ("n_tokens", ctypes.c_int64), ("window", ctypes.c_int32), ("sinks", ctypes.c_int32), ("scale", ctypes.c_float),
                ("reserved", ctypes.c_int32), ("q", ctypes.c_void_p), ("q_token_stride", ctypes.c_int64), ("q_head_stride", ctypes.c_int64),
                ("out", ctypes.c_void_p), ("out_token_stride", ctypes.c_int64), ("out_head_stride", ctypes.c_int64),
                ("seqs", ctypes.c_void_p), ("starts", ctypes.c_void_p)]


_P, _I, _L = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
# name -> (restype, argtypes); also the list the symbol test checks against the header
SIGNATURES = {
    "ic_kv_create": (_P, [ctypes.POINTER(ic_kv_opts_t)]),
    "ic_kv_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(ic_kv_opts_t)]),
    "ic_kv_reserve": (ctypes.c_int, [_P, _P, _P, _I]),
    "ic_kv_write": (ctypes.c_int, [_P, _I, _P, _P, _L, _L, _P, _P, _I, _L]),
    "ic_kv_attend": (ctypes.c_int, [_P, ctypes.POINTER(ic_kv_attend_t)]),
    "ic_kv_fork": (ctypes.c_int, [_P, _P, _P, _P, _I, _I]),
    "ic_kv_free": (ctypes.c_int, [_P, _P, _I]),
    "ic_kv_compact": (ctypes.c_int, [_P]),
    "ic_kv_sync": (ctypes.c_int, [_P]),
    "ic_kv_set_stream": (ctypes.c_int, [_P, _P]),
    "ic_kv_launch_count": (ctypes.c_int64, [_P]),
    "ic_kv_destroy": (None, [_P]),
}

_ready = None


def _library():
    global _ready
    if _ready is None:
        lib = binding.load_library()
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _ready = lib
    return _ready


def _options(n_pages, n_layers, n_kv_heads, page_size, head_dim, max_seqs, max_pages, dtype) -> ic_kv_opts_t:
    if dtype not in (torch.bfloat16, torch.float16):
        raise TypeError("dtype must be torch.bfloat16 or torch.float16")
    o = ic_kv_opts_t()
    o.struct_size = ctypes.sizeof(ic_kv_opts_t)
    o.device = -1
    o.dtype = IC_KV_F16 if dtype == torch.float16 else IC_KV_BF16
    o.n_pages, o.n_layers, o.n_kv_heads, o.page_size, o.head_dim = n_pages, n_layers, n_kv_heads, page_size, head_dim
    o.max_seqs, o.max_pages = max_seqs, max_pages
    return o


def ic_kv_workspace_bytes(n_pages: int, n_layers: int, n_kv_heads: int, page_size: int, head_dim: int, max_seqs: int,
                          max_pages: int, dtype: torch.dtype = torch.bfloat16) -> int:
    """Bytes of the `workspace` tensor for a cache of these sizes; 0 if they are invalid."""
    return int(_library().ic_kv_workspace_bytes(ctypes.byref(
        _options(n_pages, n_layers, n_kv_heads, page_size, head_dim, max_seqs, max_pages, dtype))))


class ICPagedKV:
    """Keys and values in shared pages (include/ic_kv.h).

    pool    [n_pages, n_layers, 2, n_kv_heads, page_size, head_dim]  keys at index 0, values at 1
    tables  [max_seqs, max_pages] int32, lengths [max_seqs] int32, refs [n_pages] int32

    The tensors may be given (an earlier cache's, or zeroed books); they are kept alive and used in
    place.  All index arguments are int32 device tensors.  Calls are stream ordered: made under another
    current stream than the handle's they wait for that stream and it waits for them.  What only the
    device can see wrong (IC_ERR_FULL, IC_ERR_INVALID) is raised by sync() or by a later call."""

    def __init__(self, n_pages: int, n_layers: int, n_kv_heads: int, page_size: int, head_dim: int, max_seqs: int, max_pages: int, *,
                 dtype: torch.dtype = torch.bfloat16, pool: Optional[torch.Tensor] = None, tables: Optional[torch.Tensor] = None,
                 lengths: Optional[torch.Tensor] = None, refs: Optional[torch.Tensor] = None, device: Optional[int] = None,
                 stream: Optional[torch.cuda.Stream] = None, workspace: Optional[torch.Tensor] = None):
        lib = _library()
        o = _options(n_pages, n_layers, n_kv_heads, page_size, head_dim, max_seqs, max_pages, dtype)
        if not lib.ic_kv_workspace_bytes(ctypes.byref(o)):
            raise ICCacheError(IC_ERR_INVALID, ic_cache_last_error())
        self.n_pages, self.n_layers, self.n_kv_heads, self.page_size, self.head_dim = n_pages, n_layers, n_kv_heads, page_size, head_dim
        self.max_seqs, self.max_pages, self.dtype = max_seqs, max_pages, dtype
        dev = torch.cuda.current_device() if device is None else device
        self.device = torch.device("cuda", dev)
        self._stream = stream if stream is not None else torch.cuda.current_stream(self.device)

        def tensor(given, shape, kind, what):
            if given is None:
                make = torch.empty if what == "pool" else torch.zeros
                return make(shape, dtype=kind, device=self.device)
            if tuple(given.shape) != shape or given.dtype != kind or given.device != self.device or not given.is_contiguous():
                raise ValueError(f"{what} must be a contiguous {kind} tensor of shape {list(shape)} on {self.device}")
            return given
        self.pool = tensor(pool, (n_pages, n_layers, 2, n_kv_heads, page_size, head_dim), dtype, "pool")
        self.tables = tensor(tables, (max_seqs, max_pages), torch.int32, "tables")
        self.lengths = tensor(lengths, (max_seqs,), torch.int32, "lengths")
        self.refs = tensor(refs, (n_pages,), torch.int32, "refs")
        o.device, o.stream = dev, self._stream.cuda_stream or None
        o.pool, o.tables, o.lengths, o.refs = (t.data_ptr() for t in (self.pool, self.tables, self.lengths, self.refs))
        if workspace is None:       # from torch's allocator, which has it ready more often than not
            workspace = torch.empty(lib.ic_kv_workspace_bytes(ctypes.byref(o)), dtype=torch.uint8, device=self.device)
            workspace.record_stream(self._stream)
            made = True
        else:
            made = pool is None or tables is None or lengths is None or refs is None
            if not workspace.is_cuda or not workspace.is_contiguous():
                raise ValueError("workspace must be a contiguous device tensor")
        o.workspace, o.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
        self._workspace = workspace     # borrowed by the handle: keep it alive
        if made:
            # what was made here is made before the handle's stream uses it
            self._stream.wait_stream(torch.cuda.current_stream(self.device))
        self._h = lib.ic_kv_create(ctypes.byref(o))
        if not self._h:
            self._h = None
            raise ICCacheError(IC_ERR_INVALID, ic_cache_last_error())
        self._lib = lib
        self._raw, self._index = self._stream.cuda_stream, dev
        self._a = ic_kv_attend_t()
        self._a.struct_size = ctypes.sizeof(ic_kv_attend_t)
        self._ref = ctypes.byref(self._a)
        self._scale = 1.0 / math.sqrt(head_dim)

    # -- lifetime
    def close(self) -> None:
        if getattr(self, "_h", None):
            self._lib.ic_kv_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    # -- calls
    def _call(self, fn, args, *tensors) -> None:
        if self._h is None:
            raise ValueError("the cache is closed")
        if torch._C._cuda_getCurrentRawStream(self._index) == self._raw:
            rc = fn(self._h, *args)
        else:
            # under another stream: the handle's stream takes its turn between that stream's work
            here = torch.cuda.current_stream(self.device)
            self._stream.wait_stream(here)
            rc = fn(self._h, *args)
            for t in tensors:
                if t is not None:
                    t.record_stream(self._stream)
            here.wait_stream(self._stream)
        if rc != IC_OK:
            raise ICCacheError(rc, ic_cache_last_error())

    def _ints(self, t: torch.Tensor, n: int, what: str) -> None:
        if t.dtype != torch.int32 or t.dim() != 1 or t.shape[0] != n or t.device != self.device or not t.is_contiguous():
            raise ValueError(f"{what} must be a contiguous int32 tensor of {n} entries on {self.device}")

    def _rows(self, t: torch.Tensor, what: str) -> torch.Tensor:
        """t as the kernels take it: [tokens, heads, head_dim], rows of head_dim contiguous values, 16-byte aligned, strides in
        steps of 8 elements; a copy where it is not laid out so."""
        if t.dtype != self.dtype or t.dim() != 3 or t.shape[2] != self.head_dim or t.device != self.device:
            raise ValueError(f"{what} must be a [tokens, heads, {self.head_dim}] tensor of {self.dtype} on {self.device}")
        a, b, c = t.stride()
        if (c != 1 and self.head_dim > 1) or a % 8 or b % 8 or t.data_ptr() % 16:
            t = torch.empty(t.shape, dtype=t.dtype, device=t.device).copy_(t)
        return t

    def reserve(self, seqs: torch.Tensor, counts: torch.Tensor) -> None:
        """Make room for counts[i] new tokens at the end of sequence seqs[i]."""
        n = seqs.shape[0]
        self._ints(seqs, n, "seqs")
        self._ints(counts, n, "counts")
        self._call(self._lib.ic_kv_reserve, (seqs.data_ptr(), counts.data_ptr(), n), seqs, counts)

    def write(self, layer: int, k: torch.Tensor, v: torch.Tensor, seqs: torch.Tensor, starts: Optional[torch.Tensor] = None) -> None:
        """Store the keys and values [tokens, n_kv_heads, head_dim] of each sequence's newest tokens in one layer.  starts: [n + 1],
        where a sequence's tokens begin in k and v; None = one token per sequence."""
        n = seqs.shape[0]
        self._ints(seqs, n, "seqs")
        if starts is not None:
            self._ints(starts, n + 1, "starts")
        k, v = self._rows(k, "k"), self._rows(v, "v")
        tokens, heads, _ = k.shape
        if heads != self.n_kv_heads or v.shape != k.shape:
            raise ValueError(f"k and v must have the same shape [tokens, {self.n_kv_heads}, {self.head_dim}]")
        strides = k.stride()
        if strides != v.stride():
            k, v = (torch.empty(x.shape, dtype=x.dtype, device=x.device).copy_(x) for x in (k, v))
            strides = k.stride()
        self._call(self._lib.ic_kv_write, (layer, k.data_ptr(), v.data_ptr(), strides[0], strides[1], seqs.data_ptr(),
                                           starts.data_ptr() if starts is not None else None, n, tokens), k, v, seqs, starts)

    def _attend(self, layer, q, seqs, starts, window, sinks, scale, out):
        n = seqs.shape[0]
        self._ints(seqs, n, "seqs")
        q = self._rows(q, "q")
        tokens, heads, _ = q.shape
        a = self._a
        if out is None:      # (empty_like is the quicker one, where it gives what is wanted)
            given = out = torch.empty_like(q) if q.is_contiguous() else torch.empty(q.shape, dtype=q.dtype, device=q.device)
        else:
            if out.shape != q.shape:
                raise ValueError("out must have the shape of q")
            given, out = out, self._rows(out, "out")
        a.layer, a.n, a.n_heads, a.n_tokens = layer, n, heads, tokens
        a.window, a.sinks, a.scale = window, sinks, self._scale if scale is None else scale
        a.q, (a.q_token_stride, a.q_head_stride, _) = q.data_ptr(), q.stride()
        a.out, (a.out_token_stride, a.out_head_stride, _) = out.data_ptr(), out.stride()
        a.seqs, a.starts = seqs.data_ptr(), starts.data_ptr() if starts is not None else None
        self._call(self._lib.ic_kv_attend, (self._ref,), q, out, seqs, starts)
        if out is not given:
            given.copy_(out)
        return given

    def decode(self, layer: int, q: torch.Tensor, seqs: torch.Tensor, *, window: int = 0, sinks: int = 0,
               scale: Optional[float] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Attention of the newest token of each sequence: q [n, n_heads, head_dim] -> the same shape.  out may be q; its rows may
        not overlap otherwise."""
        if q.shape[0] != seqs.shape[0]:
            raise ValueError("decode takes one token per sequence: use extend for more")
        return self._attend(layer, q, seqs, None, window, sinks, scale, out)

    def extend(self, layer: int, q: torch.Tensor, seqs: torch.Tensor, starts: torch.Tensor, *, window: int = 0, sinks: int = 0,
               scale: Optional[float] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Causal attention of each sequence's newest starts[i + 1] - starts[i] tokens: q [tokens, n_heads, head_dim] -> the same
        shape.  A token at position p sees the keys j <= p with j > p - window (window 0: all of them) or j < sinks.  out: as for
        decode."""
        self._ints(starts, seqs.shape[0] + 1, "starts")
        return self._attend(layer, q, seqs, starts, window, sinks, scale, out)

    def fork(self, parents: torch.Tensor, children: torch.Tensor, upto: Optional[torch.Tensor] = None, *, copy: bool = False) -> None:
        """Sequence children[i] becomes the first upto[i] tokens (None: all) of parents[i], all at once; full pages are shared, or
        with copy=True every page is copied."""
        n = parents.shape[0]
        self._ints(parents, n, "parents")
        self._ints(children, n, "children")
        if upto is not None:
            self._ints(upto, n, "upto")
        self._call(self._lib.ic_kv_fork, (parents.data_ptr(), children.data_ptr(), upto.data_ptr() if upto is not None else None, n,
                                          int(bool(copy))), parents, children, upto)

    def free(self, seqs: torch.Tensor) -> None:
        """Give back the pages of these sequences."""
        n = seqs.shape[0]
        self._ints(seqs, n, "seqs")
        self._call(self._lib.ic_kv_free, (seqs.data_ptr(), n), seqs)

    def compact(self) -> None:
        """Move the live pages to the front of the pool."""
        self._call(self._lib.ic_kv_compact, ())

    def sync(self) -> None:
        """Synchronise and raise (and clear) what the kernels found wrong."""
        rc = self._lib.ic_kv_sync(self._h)
        if rc != IC_OK:
            raise ICCacheError(rc, ic_cache_last_error())

    def set_stream(self, stream: torch.cuda.Stream) -> None:
        """Bind the handle to another stream, which waits for the present one."""
        stream.wait_stream(self._stream)
        rc = self._lib.ic_kv_set_stream(self._h, stream.cuda_stream or None)
        if rc != IC_OK:
            raise ICCacheError(rc, ic_cache_last_error())
        self._stream, self._raw = stream, stream.cuda_stream

    @property
    def launch_count(self) -> int:
        return int(self._lib.ic_kv_launch_count(self._h))
