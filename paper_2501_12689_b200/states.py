"""Thin ctypes binding of the state cache's C ABI (include/ic_state.h).

Argument checks and marshalling only: every step runs in the CUDA library, torch provides device
memory and streams.  `ICStates` owns a handle together with its tensors.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional

import torch

from . import binding
from .binding import IC_ERR_INVALID, IC_OK, ICCacheError, ic_cache_last_error

IC_STATE_BF16, IC_STATE_F16 = 0, 1
IC_STATE_MAX_KEY_DIM, IC_STATE_MAX_VALUE_DIM, IC_STATE_MAX_SEQS = 128, 256, 8192


class ic_state_opts_t(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32)] + [(n, ctypes.c_int32) for n in (
        "device", "dtype", "n_layers", "n_heads", "key_dim", "value_dim", "max_seqs")] + [
        (n, ctypes.c_void_p) for n in ("pool", "stream", "workspace")] + [("workspace_bytes", ctypes.c_size_t)]


class ic_state_attend_t(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("layer", ctypes.c_int32), ("n", ctypes.c_int32), ("scale", ctypes.c_float),
                ("n_tokens", ctypes.c_int64)] + [f for x in ("q", "k", "v", "out") for f in (
                    (x, ctypes.c_void_p), (x + "_token_stride", ctypes.c_int64), (x + "_head_stride", ctypes.c_int64))] + [
                        (n, ctypes.c_void_p) for n in ("rates", "seqs", "starts")]


_P, _I = ctypes.c_void_p, ctypes.c_int32
# name -> (restype, argtypes); also the list the symbol test checks against the header
SIGNATURES = {
    "ic_state_create": (_P, [ctypes.POINTER(ic_state_opts_t)]),
    "ic_state_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(ic_state_opts_t)]),
    "ic_state_attend": (ctypes.c_int, [_P, ctypes.POINTER(ic_state_attend_t)]),
    "ic_state_fork": (ctypes.c_int, [_P, _P, _P, _I]),
    "ic_state_clear": (ctypes.c_int, [_P, _P, _I]),
    "ic_state_sync": (ctypes.c_int, [_P]),
    "ic_state_set_stream": (ctypes.c_int, [_P, _P]),
    "ic_state_launch_count": (ctypes.c_int64, [_P]),
    "ic_state_destroy": (None, [_P]),
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


def _options(n_layers, n_heads, key_dim, value_dim, max_seqs, dtype) -> ic_state_opts_t:
    if dtype not in (torch.bfloat16, torch.float16):
        raise TypeError("dtype must be torch.bfloat16 or torch.float16")
    o = ic_state_opts_t()
    o.struct_size = ctypes.sizeof(ic_state_opts_t)
    o.device = -1
    o.dtype = IC_STATE_F16 if dtype == torch.float16 else IC_STATE_BF16
    o.n_layers, o.n_heads, o.key_dim, o.value_dim, o.max_seqs = n_layers, n_heads, key_dim, value_dim, max_seqs
    return o


def ic_state_workspace_bytes(n_layers: int, n_heads: int, key_dim: int, value_dim: int, max_seqs: int,
                             dtype: torch.dtype = torch.bfloat16) -> int:
    """Bytes of the `workspace` tensor for states of these sizes; 0 if they are invalid."""
    return int(_library().ic_state_workspace_bytes(ctypes.byref(_options(n_layers, n_heads, key_dim, value_dim, max_seqs, dtype))))


class ICStates:
    """States of linear attention with a decay per head (include/ic_state.h).

    pool    [max_seqs, n_layers, n_heads, key_dim, value_dim] float32; zeros for a sequence that has seen nothing

    The pool may be given; it is kept alive and used in place.  All index arguments are int32 device
    tensors.  Calls are stream ordered: made under another current stream than the handle's they wait
    for that stream and it waits for them.  What only the device can see wrong (IC_ERR_INVALID) is
    raised by sync() or by a later call."""

    def __init__(self, n_layers: int, n_heads: int, key_dim: int, value_dim: int, max_seqs: int, *, dtype: torch.dtype = torch.bfloat16,
                 pool: Optional[torch.Tensor] = None, device: Optional[int] = None, stream: Optional[torch.cuda.Stream] = None,
                 workspace: Optional[torch.Tensor] = None):
        lib = _library()
        o = _options(n_layers, n_heads, key_dim, value_dim, max_seqs, dtype)
        need = lib.ic_state_workspace_bytes(ctypes.byref(o))
        if not need:
            raise ICCacheError(IC_ERR_INVALID, ic_cache_last_error())
        self.n_layers, self.n_heads, self.key_dim, self.value_dim, self.max_seqs, self.dtype = (
            n_layers, n_heads, key_dim, value_dim, max_seqs, dtype)
        dev = torch.cuda.current_device() if device is None else device
        self.device = torch.device("cuda", dev)
        self._stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        shape = (max_seqs, n_layers, n_heads, key_dim, value_dim)
        made = pool is None or workspace is None
        if pool is None:
            pool = torch.zeros(shape, dtype=torch.float32, device=self.device)
            pool.record_stream(self._stream)
        elif tuple(pool.shape) != shape or pool.dtype != torch.float32 or pool.device != self.device or not pool.is_contiguous():
            raise ValueError(f"pool must be a contiguous float32 tensor of shape {list(shape)} on {self.device}")
        self.pool = pool
        if workspace is None:       # from torch's allocator, which has it ready more often than not
            workspace = torch.empty(need, dtype=torch.uint8, device=self.device)
            workspace.record_stream(self._stream)
        elif not workspace.is_cuda or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous device tensor")
        self._workspace = workspace     # borrowed by the handle: keep it alive
        if made:
            # what was made here is made before the handle's stream uses it
            self._stream.wait_stream(torch.cuda.current_stream(self.device))
        o.device, o.stream, o.pool = dev, self._stream.cuda_stream or None, pool.data_ptr()
        o.workspace, o.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
        self._h = lib.ic_state_create(ctypes.byref(o))
        if not self._h:
            self._h = None
            raise ICCacheError(IC_ERR_INVALID, ic_cache_last_error())
        self._lib = lib
        self._raw, self._index = self._stream.cuda_stream, dev
        self._a = ic_state_attend_t()
        self._a.struct_size = ctypes.sizeof(ic_state_attend_t)
        self._ref = ctypes.byref(self._a)
        self._scale = 1.0 / math.sqrt(key_dim)

    # -- lifetime
    def close(self) -> None:
        if getattr(self, "_h", None):
            self._lib.ic_state_destroy(self._h)
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
            raise ValueError("the states are closed")
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

    def _rows(self, t: torch.Tensor, tokens: int, dim: int, what: str) -> torch.Tensor:
        """t as the kernels take it: [tokens, n_heads, dim], rows of dim contiguous values, 16-byte aligned, strides in steps of 8
        elements; a copy where it is not laid out so."""
        if t.dtype != self.dtype or tuple(t.shape) != (tokens, self.n_heads, dim) or t.device != self.device:
            raise ValueError(f"{what} must be a [{tokens}, {self.n_heads}, {dim}] tensor of {self.dtype} on {self.device}")
        a, b, c = t.stride()
        if c != 1 or a % 8 or b % 8 or t.data_ptr() % 16:
            t = torch.empty(t.shape, dtype=t.dtype, device=t.device).copy_(t)
        return t

    def _attend(self, layer, q, k, v, rates, seqs, starts, scale, out):
        tokens, n = q.shape[0], seqs.shape[0]
        self._ints(seqs, n, "seqs")
        if rates.dtype != torch.float32 or tuple(rates.shape) != (self.n_heads,) or rates.device != self.device or not rates.is_contiguous():
            raise ValueError(f"rates must be a contiguous float32 tensor of {self.n_heads} entries on {self.device}")
        q, k, v = self._rows(q, tokens, self.key_dim, "q"), self._rows(k, tokens, self.key_dim, "k"), self._rows(v, tokens, self.value_dim, "v")
        if out is None:
            given = out = torch.empty((tokens, self.n_heads, self.value_dim), dtype=self.dtype, device=self.device)
        else:
            given, out = out, self._rows(out, tokens, self.value_dim, "out")
        a = self._a
        a.layer, a.n, a.n_tokens, a.scale = layer, n, tokens, self._scale if scale is None else scale
        a.q, (a.q_token_stride, a.q_head_stride, _) = q.data_ptr(), q.stride()
        a.k, (a.k_token_stride, a.k_head_stride, _) = k.data_ptr(), k.stride()
        a.v, (a.v_token_stride, a.v_head_stride, _) = v.data_ptr(), v.stride()
        a.out, (a.out_token_stride, a.out_head_stride, _) = out.data_ptr(), out.stride()
        a.rates, a.seqs, a.starts = rates.data_ptr(), seqs.data_ptr(), starts.data_ptr() if starts is not None else None
        self._call(self._lib.ic_state_attend, (self._ref,), q, k, v, out, rates, seqs, starts)
        if out is not given:
            given.copy_(out)
        return given

    def decode(self, layer: int, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, rates: torch.Tensor, seqs: torch.Tensor, *,
               scale: Optional[float] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """One new token of each sequence: q, k [n, n_heads, key_dim], v [n, n_heads, value_dim] -> [n, n_heads, value_dim]; the states are
        brought up to date.  rates [n_heads] float32: a token's weight falls by e ** -rate per token.  scale: 1 / sqrt(key_dim) if None."""
        if q.shape[0] != seqs.shape[0]:
            raise ValueError("decode takes one token per sequence: use extend for more")
        return self._attend(layer, q, k, v, rates, seqs, None, scale, out)

    def extend(self, layer: int, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, rates: torch.Tensor, seqs: torch.Tensor,
               starts: torch.Tensor, *, scale: Optional[float] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The newest starts[i + 1] - starts[i] tokens of each sequence: as decode, with tokens in place of n."""
        self._ints(starts, seqs.shape[0] + 1, "starts")
        return self._attend(layer, q, k, v, rates, seqs, starts, scale, out)

    def fork(self, parents: torch.Tensor, children: torch.Tensor) -> None:
        """Sequence children[i] gets the state of parents[i], all at once."""
        n = parents.shape[0]
        self._ints(parents, n, "parents")
        self._ints(children, n, "children")
        self._call(self._lib.ic_state_fork, (parents.data_ptr(), children.data_ptr(), n), parents, children)

    def clear(self, seqs: torch.Tensor) -> None:
        """These sequences have seen nothing."""
        n = seqs.shape[0]
        self._ints(seqs, n, "seqs")
        self._call(self._lib.ic_state_clear, (seqs.data_ptr(), n), seqs)

    def sync(self) -> None:
        """Synchronise and raise (and clear) what the kernels found wrong."""
        rc = self._lib.ic_state_sync(self._h)
        if rc != IC_OK:
            raise ICCacheError(rc, ic_cache_last_error())

    def set_stream(self, stream: torch.cuda.Stream) -> None:
        """Bind the handle to another stream, which waits for the present one."""
        stream.wait_stream(self._stream)
        rc = self._lib.ic_state_set_stream(self._h, stream.cuda_stream or None)
        if rc != IC_OK:
            raise ICCacheError(rc, ic_cache_last_error())
        self._stream, self._raw = stream, stream.cuda_stream

    @property
    def launch_count(self) -> int:
        return int(self._lib.ic_state_launch_count(self._h))
