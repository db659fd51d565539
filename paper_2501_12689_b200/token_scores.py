"""Thin ctypes binding of the token scores' C ABI (include/ic_score.h).

Argument checks and marshalling only: every step runs in the CUDA library, torch provides device
memory and streams.  `ICTokenScores` owns a handle.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

import torch

from . import binding
from .binding import IC_ERR_INVALID, IC_OK, ICCacheError, ic_cache_last_error

IC_SCORE_BF16, IC_SCORE_F16, IC_SCORE_F32 = 0, 1, 2
IC_SCORE_MAX_TOP, IC_SCORE_MAX_VOCAB = 32, 16777216
_DTYPES = {torch.bfloat16: IC_SCORE_BF16, torch.float16: IC_SCORE_F16, torch.float32: IC_SCORE_F32}


class ic_score_opts_t(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("device", ctypes.c_int32), ("dtype", ctypes.c_int32), ("vocab", ctypes.c_int32),
                ("stream", ctypes.c_void_p), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class ic_score_args_t(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("n_top", ctypes.c_int32), ("n_rows", ctypes.c_int64), ("scale", ctypes.c_float),
                ("reserved", ctypes.c_int32), ("logits", ctypes.c_void_p), ("row_stride", ctypes.c_int64), ("targets", ctypes.c_void_p),
                ("log_probs", ctypes.c_void_p), ("entropy", ctypes.c_void_p), ("top_ids", ctypes.c_void_p), ("top_log_probs", ctypes.c_void_p)]


_P = ctypes.c_void_p
# name -> (restype, argtypes); also the list the symbol test checks against the header
SIGNATURES = {
    "ic_score_create": (_P, [ctypes.POINTER(ic_score_opts_t)]),
    "ic_score_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(ic_score_opts_t)]),
    "ic_score_tokens": (ctypes.c_int, [_P, ctypes.POINTER(ic_score_args_t)]),
    "ic_score_sync": (ctypes.c_int, [_P]),
    "ic_score_set_stream": (ctypes.c_int, [_P, _P]),
    "ic_score_launch_count": (ctypes.c_int64, [_P]),
    "ic_score_destroy": (None, [_P]),
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


def _options(vocab: int, dtype: torch.dtype) -> ic_score_opts_t:
    if dtype not in _DTYPES:
        raise TypeError("dtype must be torch.bfloat16, torch.float16 or torch.float32")
    o = ic_score_opts_t()
    o.struct_size = ctypes.sizeof(ic_score_opts_t)
    o.device, o.dtype, o.vocab = -1, _DTYPES[dtype], vocab
    return o


def ic_score_workspace_bytes(vocab: int, dtype: torch.dtype = torch.bfloat16) -> int:
    """Bytes of the `workspace` tensor; 0 for an invalid vocabulary."""
    return int(_library().ic_score_workspace_bytes(ctypes.byref(_options(vocab, dtype))))


class TokenScores(NamedTuple):
    log_probs: Optional[torch.Tensor]       # [rows] float32, of the targets; None without
    entropy: Optional[torch.Tensor]         # [rows] float32; None if not wanted
    top_ids: Optional[torch.Tensor]         # [rows, n_top] int32; None if n_top is 0
    top_log_probs: Optional[torch.Tensor]   # [rows, n_top] float32


class ICTokenScores:
    """Log-probabilities of given tokens, entropy and top alternatives of rows of logits (include/ic_score.h).

    Calls are stream ordered: made under another current stream than the handle's they wait for that
    stream and it waits for them.  A target outside the vocabulary is raised by sync() or by a later call."""

    def __init__(self, vocab: int, *, dtype: torch.dtype = torch.bfloat16, device: Optional[int] = None,
                 stream: Optional[torch.cuda.Stream] = None, workspace: Optional[torch.Tensor] = None):
        lib = _library()
        o = _options(vocab, dtype)
        need = lib.ic_score_workspace_bytes(ctypes.byref(o))
        if not need:
            raise ICCacheError(IC_ERR_INVALID, ic_cache_last_error())
        self.vocab, self.dtype = vocab, dtype
        dev = torch.cuda.current_device() if device is None else device
        self.device = torch.device("cuda", dev)
        self._stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        if workspace is None:       # from torch's allocator, which has it ready more often than not
            workspace = torch.empty(need, dtype=torch.uint8, device=self.device)
            workspace.record_stream(self._stream)
            self._stream.wait_stream(torch.cuda.current_stream(self.device))
        elif not workspace.is_cuda or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous device tensor")
        self._workspace = workspace     # borrowed by the handle: keep it alive
        o.device, o.stream = dev, self._stream.cuda_stream or None
        o.workspace, o.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
        self._h = lib.ic_score_create(ctypes.byref(o))
        if not self._h:
            self._h = None
            raise ICCacheError(IC_ERR_INVALID, ic_cache_last_error())
        self._lib = lib
        self._raw, self._index = self._stream.cuda_stream, dev
        self._a = ic_score_args_t()
        self._a.struct_size = ctypes.sizeof(ic_score_args_t)
        self._ref = ctypes.byref(self._a)

    # -- lifetime
    def close(self) -> None:
        if getattr(self, "_h", None):
            self._lib.ic_score_destroy(self._h)
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
    def score(self, logits: torch.Tensor, targets: Optional[torch.Tensor] = None, *, n_top: int = 0, entropy: bool = True,
              scale: float = 1.0) -> TokenScores:
        """logits [rows, vocab]; targets [rows] int32 (-1: none, its log-probability is 0); scale: one over the temperature."""
        if self._h is None:
            raise ValueError("the scores are closed")
        if logits.dtype != self.dtype or logits.dim() != 2 or logits.shape[1] != self.vocab or logits.device != self.device:
            raise ValueError(f"logits must be a [rows, {self.vocab}] tensor of {self.dtype} on {self.device}")
        rows = logits.shape[0]
        if targets is not None and (targets.dtype != torch.int32 or targets.dim() != 1 or targets.shape[0] != rows
                                    or targets.device != self.device or not targets.is_contiguous()):
            raise ValueError(f"targets must be a contiguous int32 tensor of {rows} entries on {self.device}")
        if logits.stride(1) != 1 and self.vocab > 1:
            logits = logits.contiguous()
        a = self._a
        make = lambda shape, kind: torch.empty(shape, dtype=kind, device=self.device)  # noqa: E731
        log_probs = make(rows, torch.float32) if targets is not None else None
        spread = make(rows, torch.float32) if entropy else None
        ids = make((rows, n_top), torch.int32) if n_top > 0 else None
        top = make((rows, n_top), torch.float32) if n_top > 0 else None
        a.n_top, a.n_rows, a.scale = n_top, rows, scale
        a.logits, a.row_stride = logits.data_ptr(), logits.stride(0)
        a.targets, a.log_probs, a.entropy, a.top_ids, a.top_log_probs = (
            t.data_ptr() if t is not None else None for t in (targets, log_probs, spread, ids, top))
        if torch._C._cuda_getCurrentRawStream(self._index) == self._raw:
            rc = self._lib.ic_score_tokens(self._h, self._ref)
        else:
            # under another stream: the handle's stream takes its turn between that stream's work
            here = torch.cuda.current_stream(self.device)
            self._stream.wait_stream(here)
            rc = self._lib.ic_score_tokens(self._h, self._ref)
            for t in (logits, targets, log_probs, spread, ids, top):
                if t is not None:
                    t.record_stream(self._stream)
            here.wait_stream(self._stream)
        if rc != IC_OK:
            raise ICCacheError(rc, ic_cache_last_error())
        return TokenScores(log_probs, spread, ids, top)

    def sync(self) -> None:
        """Synchronise and raise (and clear) what the kernels found wrong."""
        rc = self._lib.ic_score_sync(self._h)
        if rc != IC_OK:
            raise ICCacheError(rc, ic_cache_last_error())

    def set_stream(self, stream: torch.cuda.Stream) -> None:
        """Bind the handle to another stream, which waits for the present one."""
        stream.wait_stream(self._stream)
        rc = self._lib.ic_score_set_stream(self._h, stream.cuda_stream or None)
        if rc != IC_OK:
            raise ICCacheError(rc, ic_cache_last_error())
        self._stream, self._raw = stream, stream.cuda_stream

    @property
    def launch_count(self) -> int:
        return int(self._lib.ic_score_launch_count(self._h))
