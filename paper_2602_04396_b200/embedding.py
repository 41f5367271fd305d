"""Embedding lookup with scaling and its gradient by sorted tokens (argument marshalling for include/lordo.h).

For one table, or for the K workers' replicas of one: ``W`` is [V, d] with tokens of any shape, or [K, V, d] with tokens [K, ...].
Tokens are int32 or int64; one outside [0, V) is padding: a row of zeros, and no share in the gradient. Both calls work on
the tensors' device, enqueue on ``stream`` (default: the device's current one) and can be captured in a CUDA graph. What a call allocates
belongs to its stream; with ``stream`` the tensors handed over are recorded on it, so that they may be dropped after the call.
"""
from __future__ import annotations

import ctypes as C
import functools
from typing import Optional

import torch

from .lordo import LordoError, _dtype_code, load_library, used_on

_INDEX = {torch.int32: 0, torch.int64: 1}
_raw_stream = torch._C._cuda_getCurrentRawStream  # torch.cuda.current_stream builds an object: 3 us of a call's 10


def _checked(t: torch.Tensor, what: str, index: int) -> None:
    if t.get_device() != index or index < 0 or not t.is_contiguous():
        raise ValueError(f"{what}: a contiguous CUDA tensor on the call's device is wanted")


def _tokens_per_worker(tokens: torch.Tensor, K: int, table: bool) -> int:
    """Of tokens [K, ...], or of any shape for a single table."""
    if tokens.dtype not in _INDEX:
        raise ValueError(f"tokens: int32 or int64 is wanted, not {tokens.dtype}")
    if table and (tokens.dim() < 2 or tokens.shape[0] != K):
        raise ValueError(f"tokens: [K, ...] with K = {K} is wanted, not {tuple(tokens.shape)}")
    if K < 1:
        raise ValueError("at least one worker is wanted")
    return tokens.numel() // K


def _on(index: int, stream: Optional[torch.cuda.Stream]):
    """A context with the device current, and `stream` too where one is given, so that what is allocated belongs to it; None where it is so already."""
    if stream is not None:
        if stream.device.index != index:
            raise ValueError(f"stream: one of device {index} is wanted, not of {stream.device}")
        return torch.cuda.stream(stream)
    return None if index == torch.cuda.current_device() else torch.cuda.device(index)


@functools.lru_cache(maxsize=256)
def _workspace(K: int, V: int, d: int, T: int) -> int:
    need = C.c_size_t(0)
    lib = load_library()
    rc = lib.lordo_embedding_grad_query_workspace(K, V, d, T, C.byref(need))
    if rc != 0:
        raise LordoError(rc, "lordo_embedding_grad_query_workspace", lib.lordo_status_string(rc).decode())
    return need.value


def embedding(W: torch.Tensor, tokens: torch.Tensor, *, scale: float = 1.0, out: Optional[torch.Tensor] = None,
              out_dtype: Optional[torch.dtype] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """scale * W[token], of shape tokens.shape + (d,) and of W's dtype unless ``out`` or ``out_dtype`` says otherwise. No part of autograd: a
    table that requires a gradient is refused where one would be recorded (W.detach(), or a torch.autograd.Function around both calls)."""
    device = W.get_device()
    context = _on(device, stream) if device >= 0 else None
    if context is not None:
        with context:
            result = embedding(W, tokens, scale=scale, out=out, out_dtype=out_dtype)
        if stream is not None:
            used_on(stream, W, tokens, out)
        return result
    _checked(W, "W", device)
    _checked(tokens, "tokens", device)
    if W.requires_grad and torch.is_grad_enabled():
        raise ValueError("W requires a gradient, which the lookup does not record: W.detach() and embedding_grad are wanted")
    if W.dim() not in (2, 3):
        raise ValueError("W: [V, d] or [K, V, d] is wanted")
    V, d = W.shape[-2:]
    K = W.shape[0] if W.dim() == 3 else 1
    T = _tokens_per_worker(tokens, K, W.dim() == 3)
    shape = tokens.shape + (d,)
    if out is None:
        out = torch.empty(shape, device=W.device, dtype=out_dtype or W.dtype)
    else:
        _checked(out, "out", device)
        if out.shape != shape or (out_dtype is not None and out.dtype != out_dtype):
            raise ValueError(f"out: {tuple(shape)} is wanted, not {tuple(out.shape)}, or its dtype is not out_dtype")
    lib = load_library()
    rc = lib.lordo_embedding(W.data_ptr(), _dtype_code(W.dtype), K, V, d, tokens.data_ptr(), _INDEX[tokens.dtype], T, scale, out.data_ptr(),
                             _dtype_code(out.dtype), _raw_stream(device))
    if rc != 0:
        raise LordoError(rc, "lordo_embedding", lib.lordo_status_string(rc).decode())
    return out


def embedding_grad(dY: torch.Tensor, tokens: torch.Tensor, V: int, *, scale: float = 1.0, out: Optional[torch.Tensor] = None,
                   out_dtype: Optional[torch.dtype] = None, accumulate: bool = False, K: Optional[int] = None,
                   stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """The table's gradient, [V, d], or [K, V, d] where ``out`` has three dimensions or ``K`` is given: scale times the sum of the
    rows of dY (tokens.shape + (d,)) that belong to each token. ``accumulate`` adds it to ``out`` and leaves rows without a token as
    they are. Sums are formed in fp32, the same bits on every run."""
    device = dY.get_device()
    context = _on(device, stream) if device >= 0 else None
    if context is not None:
        with context:
            result = embedding_grad(dY, tokens, V, scale=scale, out=out, out_dtype=out_dtype, accumulate=accumulate, K=K)
        if stream is not None:
            used_on(stream, dY, tokens, out)
        return result
    _checked(dY, "dY", device)
    _checked(tokens, "tokens", device)
    d = dY.shape[-1]
    if out is not None:
        _checked(out, "out", device)
        if out.dim() not in (2, 3) or out.shape[-2:] != (V, d) or (out.dim() == 3 and K not in (None, out.shape[0])) or (out.dim() == 2 and K is not None):
            raise ValueError(f"out: [V, d] or [K, V, d] is wanted, not {tuple(out.shape)}")
        if out_dtype is not None and out.dtype != out_dtype:
            raise ValueError("out: its dtype is not out_dtype")
        K = out.shape[0] if out.dim() == 3 else None
    elif accumulate:
        raise ValueError("accumulate needs an out to add to")
    workers = 1 if K is None else K
    if dY.shape != tokens.shape + (d,):
        raise ValueError(f"dY: {tuple(tokens.shape)} + (d,) is wanted, not {tuple(dY.shape)}")
    T = _tokens_per_worker(tokens, workers, K is not None)
    need = _workspace(workers, V, d, T)
    if out is None:
        out = torch.empty((V, d) if K is None else (K, V, d), device=dY.device, dtype=out_dtype or dY.dtype)
    workspace = torch.empty(need, device=dY.device, dtype=torch.uint8)  # torch's allocations are 512-byte aligned
    lib = load_library()
    rc = lib.lordo_embedding_grad(dY.data_ptr(), _dtype_code(dY.dtype), tokens.data_ptr(), _INDEX[tokens.dtype], workers, V, d, T, scale, out.data_ptr(),
                                  _dtype_code(out.dtype), 1 if accumulate else 0, workspace.data_ptr(), need, _raw_stream(device))
    if rc != 0:
        raise LordoError(rc, "lordo_embedding_grad", lib.lordo_status_string(rc).decode())
    return out
