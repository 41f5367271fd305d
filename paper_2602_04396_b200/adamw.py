"""AdamW for the parameters outside the low-rank path (embedding tables, norm gains, biases), K workers' replicas each
(argument marshalling for the lordo_adamw_* calls of include/lordo.h).

    matrices = lordo.Lordo(mats, K, H, W0)                       # the low-rank path
    others = adamw.AdamW(W0_others, K, states="8bit", tables={0: tokens_per_worker}, outer=lordo.OUTER_NESTEROV, ...)
    for every step:   matrices.inner_step(G, lr, beta1, omega, form)
                      others.step([adamw.TokenGrad(tokens, dY, scale), G1, G2, ...], lr, beta1)
    every H steps:    matrices.outer_step(); others.outer_step()
"""
from __future__ import annotations

import ctypes as C
from array import array
from typing import Dict, List, NamedTuple, Optional, Sequence, Union

import torch

from . import lordo
from .lordo import LordoError, _AdamWBuffers, _AdamWConfig, _Grad, _Tensor, _dtype_code, _ptr_table, load_library, used_on

_INDEX = {torch.int32: 0, torch.int64: 1}
_STATES = {"f32": 0, "8bit": 1}
_raw_stream = torch._C._cuda_getCurrentRawStream  # without the object that torch.cuda.current_stream builds
BLOCK = 256  # elements per scale of the 8-bit moments


class TokenGrad(NamedTuple):
    """A table's gradient in the form of its lookup's: tokens [K, ...] and dY of tokens.shape + (d,), the gradient of ``scale * W[token]``.
    A token outside [0, V) is padding."""
    tokens: torch.Tensor
    dY: torch.Tensor
    scale: float = 1.0


class AdamW:
    """Owns the device arrays of one group (through PyTorch) and forwards the calls to the library.

    W0: tensors of any shape in the weight dtype. ``storage`` holds each kind of array as one flat tensor: "W", "m", "v" (each
    tensor's [K][n] from a multiple of 128 elements on), with 8-bit moments "ms", "vs" (their scales, [K][ceil(n / 256)]), with
    ``outer`` "X0", "B" ([n]); ``W[i]`` and the like are views of one tensor, [K, *shape] (scales [K, blocks], X0 and B [*shape]).
    With ``get_counters`` they are all that a checkpoint needs.

    states: "f32", or "8bit" (m and sqrt(v) as float8_e4m3fn codes with float8_e8m0fnu scales, rounded at random from ``seed``).
    weight_decay: one number, or one per tensor. tables: {tensor: most tokens of a worker in a step} for the two-dimensional tensors
    whose gradient comes as TokenGrad. outer: lordo.OUTER_AVG or lordo.OUTER_NESTEROV, or None for a group that is not synchronised.
    """

    def __init__(self, W0: Sequence[torch.Tensor], K: int, *, device: str = "cuda", g_dtype: Optional[torch.dtype] = None, states: str = "f32",
                 weight_decay: Union[float, Sequence[float]] = 0.0, beta2: float = 0.999, eps: float = 1e-8, clip_rho: float = 0.0,
                 clip_scope: int = 0, outer: Optional[int] = None, outer_lr: float = 1.0, outer_momentum: float = 0.0, sync_m: bool = True,
                 sync_v: bool = True, seed: int = 0, tables: Optional[Dict[int, int]] = None):
        self._ctx = C.c_void_p(None)
        self.lib = load_library()
        if not W0:
            raise ValueError("W0: at least one tensor is wanted")
        if states not in _STATES:
            raise ValueError(f"states: one of {sorted(_STATES)} is wanted")
        w_dtype = W0[0].dtype
        if any(w.dtype != w_dtype or w.numel() == 0 for w in W0):
            raise ValueError("W0: tensors of one dtype that are not empty are wanted")
        self.K, self.states, self.outer = int(K), states, outer
        self.shapes = [tuple(w.shape) for w in W0]
        self.w_dtype, self.g_dtype = w_dtype, g_dtype or w_dtype
        self.tables = dict(tables or {})
        dev = torch.device(device)
        self.device = torch.device(dev.type, torch.cuda.current_device()) if dev.index is None else dev
        decay = [float(weight_decay)] * len(W0) if isinstance(weight_decay, (int, float)) else [float(x) for x in weight_decay]
        if len(decay) != len(W0):
            raise ValueError("weight_decay: one number, or one per tensor, is wanted")
        n = [w.numel() for w in W0]
        for i, most in self.tables.items():
            if not 0 <= i < len(W0) or len(self.shapes[i]) != 2 or most < 0:
                raise ValueError("tables: {number of a two-dimensional tensor: most tokens} is wanted")
        self._tensors = (_Tensor * len(n))(*[
            _Tensor(c, self.shapes[i][1] if i in self.tables else 0, self.tables.get(i, 0), decay[i]) for i, c in enumerate(n)])
        small = states == "8bit"
        self.cfg = _AdamWConfig(len(n), self._tensors, self.K, _dtype_code(w_dtype), _dtype_code(self.g_dtype), _STATES[states], beta2, eps, clip_rho,
                                clip_scope, int(outer is not None), int(sync_m), int(sync_v), lordo.OUTER_AVG if outer is None else outer,
                                outer_lr, outer_momentum, seed)
        need = C.c_size_t(0)
        rc = self.lib.lordo_adamw_query_workspace(C.byref(self.cfg), C.byref(need))
        if rc != 0:
            raise LordoError(rc, "lordo_adamw_query_workspace", self.lib.lordo_status_string(rc).decode())

        moment = torch.float8_e4m3fn if small else torch.float32
        blocks = [(c + BLOCK - 1) // BLOCK for c in n]
        kinds = [("W", w_dtype, n, True), ("m", moment, n, True), ("v", moment, n, True)]
        if small:
            kinds += [("ms", torch.float8_e8m0fnu, blocks, True), ("vs", torch.float8_e8m0fnu, blocks, True)]
        if outer is not None:
            kinds += [("X0", torch.float32, n, False), ("B", torch.float32, n, False)]
        self.storage: Dict[str, torch.Tensor] = {}
        views: Dict[str, List[torch.Tensor]] = {name: [] for name in ("W", "m", "v", "ms", "vs", "X0", "B")}
        with torch.cuda.device(self.device):
            for name, dtype, counts, replicas in kinds:
                sizes = [c * (self.K if replicas else 1) for c in counts]
                at = [0]
                for s in sizes:
                    at.append(at[-1] + (s + 127) // 128 * 128)
                width = torch.empty((), dtype=dtype).element_size()
                flat = torch.zeros(at[-1] * width, device=self.device, dtype=torch.uint8).view(dtype)
                self.storage[name] = flat
                for i, (o, s) in enumerate(zip(at, sizes)):
                    shape = (counts[i],) if name in ("ms", "vs") else self.shapes[i]
                    views[name].append(flat[o:o + s].view(((self.K,) if replicas else ()) + shape))
            self.W, self.m, self.v, self.ms, self.vs, self.X0, self.B = (views[x] for x in ("W", "m", "v", "ms", "vs", "X0", "B"))
            for w, w0 in zip(self.W, W0):
                w[0].copy_(w0.detach())  # a parameter would make the arrays part of its graph
            self._pointers = {name: _ptr_table(v, len(n)) for name, v in views.items() if v}
            bufs = _AdamWBuffers(*[C.cast(self._pointers[x], C.POINTER(C.c_void_p)) if x in self._pointers else None
                                   for x in ("W", "m", "v", "ms", "vs", "X0", "B")])
            self.workspace_bytes = need.value
            self.workspace = torch.empty(need.value, device=self.device, dtype=torch.uint8)  # 512-byte aligned
            rc = self.lib.lordo_adamw_init(C.byref(self.cfg), C.byref(bufs), self.workspace.data_ptr(), need.value,
                                           torch.cuda.current_stream().cuda_stream, C.byref(self._ctx))
        if rc != 0:
            raise LordoError(rc, "lordo_adamw_init", self.lib.lordo_status_string(rc).decode())
        self._grads = (_Grad * len(n))()
        words = memoryview(self._grads).cast("B").cast("Q")  # four to a gradient, the first two its addresses
        self._grad_at, self._tokens_at = words[0::4], words[1::4]
        self._no_tokens = memoryview(array("Q", bytes(8 * len(n))))
        self._full = [torch.Size((self.K,) + s) for s in self.shapes]

    # -- helpers -----------------------------------------------------------------------------
    def _check(self, rc: int, where: str):
        if rc != 0:
            raise LordoError(rc, where, self.lib.lordo_adamw_last_error(self._ctx).decode())

    def _stream(self, stream: Optional[torch.cuda.Stream]) -> int:
        if stream is None:
            return _raw_stream(self.device.index)
        if stream.device != self.device:
            raise ValueError(f"stream: one of {self.device} is wanted, not of {stream.device}")
        return stream.cuda_stream

    def _token_grad(self, i: int, g: TokenGrad) -> int:
        """Fills the gradient's entry but for the address of dY, which is returned."""
        tokens, dY, scale = g
        if i not in self.tables:
            raise ValueError(f"gradient {i}: tensor {i} is not among the tables")
        if tokens.dtype not in _INDEX or dY.dtype != self.g_dtype:
            raise ValueError(f"gradient {i}: tokens in int32 or int64 and dY in {self.g_dtype} are wanted")
        if tokens.dim() < 2 or tokens.shape[0] != self.K or tuple(dY.shape) != tuple(tokens.shape) + self.shapes[i][1:]:
            raise ValueError(f"gradient {i}: tokens [K, ...] and dY of their shape + (d,) are wanted")
        if tokens.device != self.device or dY.device != self.device or not tokens.is_contiguous() or not dY.is_contiguous():
            raise ValueError(f"gradient {i}: contiguous tensors on {self.device} are wanted")
        e = self._grads[i]
        e.T, e.index, e.scale = tokens.numel() // self.K, _INDEX[tokens.dtype], scale
        # an empty tensor has no address, and without tokens the gradient would be a dense one
        e.tokens = tokens.data_ptr() if e.T else self.workspace.data_ptr()
        return dY.data_ptr() if e.T else self.workspace.data_ptr()

    # -- calls -------------------------------------------------------------------------------
    def step(self, G: Sequence[Union[torch.Tensor, TokenGrad]], lr: float, beta1: float = 0.9, omega: float = 1.0,
             coef: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
        """One step. G: per tensor [K, *shape] in g_dtype, or TokenGrad. coef: K clip coefficients in device memory in place of the
        group's own (for instance those of a Lordo). All may be dropped after the call: with ``stream`` they are recorded on it. Its order with the
        streams that make them is the caller's."""
        if len(G) != len(self.shapes):
            raise ValueError(f"{len(self.shapes)} gradients are wanted, not {len(G)}")
        dt, index, at = self.g_dtype, self.device.index, array("Q")
        self._tokens_at[:] = self._no_tokens
        for g, shape in zip(G, self._full):
            if g.__class__ is TokenGrad:
                at.append(self._token_grad(len(at), g))
            elif g.shape != shape or g.dtype is not dt or g.get_device() != index or not g.is_contiguous():
                raise ValueError(f"gradient {len(at)}: a contiguous {tuple(shape)} tensor in {dt} on {self.device} is wanted")
            else:
                at.append(g.data_ptr())
        self._grad_at[:] = memoryview(at)
        if coef is not None and (coef.dtype != torch.float32 or coef.numel() != self.K or coef.device != self.device or not coef.is_contiguous()):
            raise ValueError(f"coef: {self.K} contiguous float32 values on {self.device} are wanted")
        rc = self._run(self.lib.lordo_adamw_step, self._grads, lr, beta1, omega, coef.data_ptr() if coef is not None else None, self._stream(stream))
        if stream is not None:
            for g in G:
                used_on(stream, *(g[:2] if g.__class__ is TokenGrad else (g,)))
            used_on(stream, coef)
        self._check(rc, "lordo_adamw_step")

    def _run(self, call, *args) -> int:
        """A call that launches, with the group's device current."""
        if torch.cuda.current_device() == self.device.index:
            return call(self._ctx, *args)
        with torch.cuda.device(self.device):
            return call(self._ctx, *args)

    def outer_step(self, stream: Optional[torch.cuda.Stream] = None):
        self._check(self._run(self.lib.lordo_adamw_outer_step, self._stream(stream)), "lordo_adamw_outer_step")

    def poll_status(self, stream: Optional[torch.cuda.Stream] = None) -> int:
        flags = C.c_uint32(0)
        rc = self._run(self.lib.lordo_adamw_poll_status, self._stream(stream), C.byref(flags))
        if rc not in (0, 7):
            self._check(rc, "lordo_adamw_poll_status")
        return flags.value

    def clear_status(self, stream: Optional[torch.cuda.Stream] = None):
        self._check(self._run(self.lib.lordo_adamw_clear_status, self._stream(stream)), "lordo_adamw_clear_status")

    def counters(self) -> List[int]:
        """[steps, synchronisations] done."""
        out = (C.c_int64 * 2)()
        self._check(self.lib.lordo_adamw_get_counters(self._ctx, out), "lordo_adamw_get_counters")
        return list(out)

    def set_counters(self, values: Sequence[int]):
        self._check(self.lib.lordo_adamw_set_counters(self._ctx, (C.c_int64 * 2)(*values)), "lordo_adamw_set_counters")

    def clip_coefficients(self) -> torch.Tensor:
        """[n_tensors, K] clip coefficients of the last step that formed them, copied out of the workspace on the current stream."""
        ptr = C.c_void_p(None)
        self._check(self.lib.lordo_adamw_clip_coefficients(self._ctx, C.byref(ptr)), "lordo_adamw_clip_coefficients")
        off, n = ptr.value - self.workspace.data_ptr(), len(self.shapes) * self.K
        return self.workspace[off:off + 4 * n].view(torch.float32).view(len(self.shapes), self.K).clone()

    @property
    def launch_count(self) -> int:
        return int(self.lib.lordo_adamw_launch_count(self._ctx))

    def close(self):
        if getattr(self, "_ctx", None) is not None and self._ctx.value:
            torch.cuda.synchronize(self.device)
            self.lib.lordo_adamw_destroy(self._ctx)
            self._ctx = C.c_void_p(None)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
