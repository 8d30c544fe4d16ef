"""Operators on token tables: ctypes binding of ``include/flashtokens.h``.

Argument marshalling only, as in :mod:`.kmeans`: tensors must be contiguous CUDA
(HIP) tensors on the current device, work is enqueued on torch's current stream,
and every output may be passed in.  A table is ``[V, D]`` (one instance) or
``[B, V, D]``; tokens are int32, and a token outside ``[0, V)`` is none.  The calls take
no part in autograd: gradients come from the ``_grad`` calls.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

import torch

from .kmeans import _DTYPE, KMeansError, _check, _need, lib  # noqa: F401

_i64, _i32, _vp, _sz, _f32 = (ctypes.c_int64, ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t,
                              ctypes.c_float)
lib.tokens_embed.argtypes = [_vp, _i32, _vp, _i64, _i64, _i64, _i64, _f32, _vp, _vp]
lib.tokens_embed_grad.argtypes = [_vp, _i32, _vp, _i64, _i64, _i64, _i64, _f32, _i32, _vp, _i32, _vp,
                                  _sz, _vp]
lib.tokens_logprobs.argtypes = [_vp, _vp, _i32, _vp, _vp, _i64, _i64, _i64, _i64, _f32, _i32, _vp, _vp,
                                _vp, _vp, _vp, _vp, _sz, _vp]
lib.tokens_logprobs_grad.argtypes = [_vp, _vp, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _i64, _i64, _i64,
                                     _i64, _f32, _vp, _vp, _vp, _sz, _vp]
lib.tokens_embed_grad_workspace_bytes.argtypes = [_i64, _i64, _i64, _i64, _i32]
lib.tokens_logprobs_workspace_bytes.argtypes = [_i64, _i64, _i64, _i64, _i32, _i32]
lib.tokens_logprobs_grad_workspace_bytes.argtypes = [_i64, _i64, _i64, _i64, _i32]
for _f in (lib.tokens_embed, lib.tokens_embed_grad, lib.tokens_logprobs, lib.tokens_logprobs_grad):
    _f.restype = ctypes.c_int
for _f in (lib.tokens_embed_grad_workspace_bytes, lib.tokens_logprobs_workspace_bytes,
           lib.tokens_logprobs_grad_workspace_bytes):
    _f.restype = ctypes.c_size_t


# A call of a few microseconds should not wait for its own checks: the current device and
# stream are asked for once, in the form that costs least.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _current() -> Tuple[int, Optional[int]]:
    """The current device and its stream's handle."""
    dev = torch.cuda.current_device()
    return dev, _raw_stream(dev) if _raw_stream else torch.cuda.current_stream().cuda_stream


def _dt(t: torch.Tensor, name: str) -> int:
    try:
        return _DTYPE[t.dtype]
    except KeyError:
        raise TypeError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}") from None


def _in(t: torch.Tensor, name: str, dev: int, dtype=None, numel: Optional[int] = None) -> int:
    """The address of a tensor that passes kmeans._need's checks (which report what fails)."""
    if (t.get_device() != dev or not t.is_contiguous() or (dtype is not None and t.dtype != dtype) or
            (numel is not None and t.numel() != numel)):
        _need(t, name, dtype, numel)
    return t.data_ptr()


def _rows(t: torch.Tensor, name: str) -> Tuple[int, int, int]:
    """[B, rows, D], or [rows, D] as one instance."""
    n = t.dim()
    if n not in (2, 3):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, want [rows, D] or [B, rows, D]")
    return tuple(t.shape) if n == 3 else (1, *t.shape)


def _workspace(ws: Optional[torch.Tensor], need: int, like: torch.Tensor,
               dev: int) -> Tuple[torch.Tensor, int]:
    if need == 0:  # arguments that the call rejects, and says why
        return like.new_empty(0, dtype=torch.uint8), 0
    if ws is None or ws.numel() < need:
        ws = torch.empty(need, dtype=torch.uint8, device=like.device)
    return ws, _in(ws, "ws", dev, torch.uint8)


def tokens_embed(table: torch.Tensor, idx: torch.Tensor, scale: float = 1.0,
                 out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """scale * table[idx], ``[B, M, D]``; zero rows where there is no token (see
    ``tokens_embed`` in the header)."""
    dt = _dt(table, "table")
    B, V, D = _rows(table, "table")
    dev, stream = _current()
    W = _in(table, "table", dev)
    t = _in(idx, "idx", dev, torch.int32)
    n = idx.dim()
    if n not in (1, 2) or (idx.shape[0] if n == 2 else 1) != B:
        raise ValueError(f"idx has shape {tuple(idx.shape)}, want [B, M] with B = {B}")
    M = idx.shape[-1]
    if out is None:
        out = torch.empty((B, M, D), dtype=table.dtype, device=table.device)
    _check(lib.tokens_embed(W, dt, t, B, M, V, D, scale,
                            _in(out, "out", dev, table.dtype, B * M * D), stream), "tokens_embed")
    return out


def embed_grad_workspace_bytes(B: int, M: int, V: int, D: int, dtype: torch.dtype) -> int:
    return int(lib.tokens_embed_grad_workspace_bytes(B, M, V, D, _DTYPE[dtype]))


def tokens_embed_grad(grad: torch.Tensor, idx: torch.Tensor, V: int, scale: float = 1.0,
                      out: Optional[torch.Tensor] = None, accumulate: bool = False,
                      ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The gradient of ``tokens_embed`` in the table, ``[B, V, D]`` in grad's type, or in
    that of ``out`` (grad's or float32); ``accumulate`` adds it to what ``out`` holds
    (see ``tokens_embed_grad`` in the header)."""
    dt = _dt(grad, "grad")
    B, M, D = _rows(grad, "grad")
    dev, stream = _current()
    G = _in(grad, "grad", dev)
    t = _in(idx, "idx", dev, torch.int32, B * M)
    if out is None:
        if accumulate:
            raise ValueError("accumulate adds to out: pass it in")
        out = torch.empty((B, V, D), dtype=grad.dtype, device=grad.device)
    elif out.dtype not in (grad.dtype, torch.float32):
        raise TypeError(f"out must be {grad.dtype} or float32, got {out.dtype}")
    o = _in(out, "out", dev, None, B * V * D)
    ws, w = _workspace(ws, lib.tokens_embed_grad_workspace_bytes(B, M, V, D, dt), grad, dev)
    _check(lib.tokens_embed_grad(G, dt, t, B, M, V, D, scale, int(accumulate), o, _DTYPE[out.dtype], w,
                                 ws.numel(), stream), "tokens_embed_grad")
    return out


def _scored(X: torch.Tensor, W: torch.Tensor, bias: Optional[torch.Tensor], dev: int):
    B, M, D = _rows(X, "X")
    Bw, V, Dw = _rows(W, "W")
    if B != Bw or D != Dw:
        raise ValueError(f"shapes X{tuple(X.shape)} W{tuple(W.shape)}: want [B,M,D] and [B,V,D]")
    dt = _dt(X, "X")
    if X.dtype != W.dtype:
        raise TypeError("rows and table must share a dtype")
    return (B, M, V, D, dt, _in(X, "X", dev), _in(W, "W", dev),
            None if bias is None else _in(bias, "bias", dev, torch.float32, B * V))


def logprobs_workspace_bytes(B: int, M: int, V: int, D: int, k: int, dtype: torch.dtype) -> int:
    return int(lib.tokens_logprobs_workspace_bytes(B, M, V, D, k, _DTYPE[dtype]))


def tokens_logprobs(X: torch.Tensor, W: torch.Tensor, target: Optional[torch.Tensor] = None, *,
                    k: int = 0, scale: float = 1.0, bias: Optional[torch.Tensor] = None,
                    logprob: Optional[torch.Tensor] = None, entropy: Optional[torch.Tensor] = None,
                    lse: Optional[torch.Tensor] = None, top_idx: Optional[torch.Tensor] = None,
                    top_logprob: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None):
    """(logprob, entropy, lse, top_idx, top_logprob) of the rows' softmax over the scores
    ``scale * X W^T + bias`` (see ``tokens_logprobs`` in the header).  logprob is None
    without a target, the last two with k = 0."""
    dev, stream = _current()
    B, M, V, D, dt, x, w, bz = _scored(X, W, bias, dev)
    k, f32, on = int(k), torch.float32, X.device
    t = lp = ti = tl = None
    if target is not None:
        t = _in(target, "target", dev, torch.int32, B * M)
        if logprob is None:
            logprob = torch.empty((B, M), dtype=f32, device=on)
        lp = _in(logprob, "logprob", dev, f32, B * M)
    elif logprob is not None:
        raise ValueError("logprob needs a target")
    if entropy is None:
        entropy = torch.empty((B, M), dtype=f32, device=on)
    if lse is None:
        lse = torch.empty((B, M), dtype=f32, device=on)
    if k > 0:
        if top_idx is None:
            top_idx = torch.empty((B, M, k), dtype=torch.int32, device=on)
        if top_logprob is None:
            top_logprob = torch.empty((B, M, k), dtype=f32, device=on)
        ti = _in(top_idx, "top_idx", dev, torch.int32, B * M * k)
        tl = _in(top_logprob, "top_logprob", dev, f32, B * M * k)
    elif top_idx is not None or top_logprob is not None:
        raise ValueError("top_idx and top_logprob need k > 0")
    ws, p = _workspace(ws, lib.tokens_logprobs_workspace_bytes(B, M, V, D, k, dt), X, dev)
    _check(lib.tokens_logprobs(x, w, dt, bz, t, B, M, V, D, scale, k, lp,
                               _in(entropy, "entropy", dev, f32, B * M),
                               _in(lse, "lse", dev, f32, B * M), ti, tl, p, ws.numel(), stream),
           "tokens_logprobs")
    return logprob, entropy, lse, top_idx, top_logprob


def logprobs_grad_workspace_bytes(B: int, M: int, V: int, D: int, dtype: torch.dtype) -> int:
    return int(lib.tokens_logprobs_grad_workspace_bytes(B, M, V, D, _DTYPE[dtype]))


def tokens_logprobs_grad(X: torch.Tensor, W: torch.Tensor, target: torch.Tensor, lse: torch.Tensor,
                         grad_logprob: torch.Tensor, *, entropy: Optional[torch.Tensor] = None,
                         grad_entropy: Optional[torch.Tensor] = None, scale: float = 1.0,
                         bias: Optional[torch.Tensor] = None, dX: Optional[torch.Tensor] = None,
                         dW: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None):
    """(dX, dW) of ``sum(grad_logprob * logprob + grad_entropy * entropy)``, from what
    ``tokens_logprobs`` returned (see ``tokens_logprobs_grad`` in the header)."""
    dev, stream = _current()
    B, M, V, D, dt, x, w, bz = _scored(X, W, bias, dev)
    f32, ent, h = torch.float32, None, None
    t = _in(target, "target", dev, torch.int32, B * M)
    l = _in(lse, "lse", dev, f32, B * M)
    g = _in(grad_logprob, "grad_logprob", dev, f32, B * M)
    if grad_entropy is not None:
        if entropy is None:
            raise ValueError("grad_entropy needs the entropy of the forward pass")
        h = _in(grad_entropy, "grad_entropy", dev, f32, B * M)
        ent = _in(entropy, "entropy", dev, f32, B * M)
    if dX is None:
        dX = torch.empty((B, M, D), dtype=X.dtype, device=X.device)
    if dW is None:
        dW = torch.empty((B, V, D), dtype=X.dtype, device=X.device)
    ws, p = _workspace(ws, lib.tokens_logprobs_grad_workspace_bytes(B, M, V, D, dt), X, dev)
    _check(lib.tokens_logprobs_grad(x, w, dt, bz, t, l, ent, g, h, B, M, V, D, scale,
                                    _in(dX, "dX", dev, X.dtype, B * M * D),
                                    _in(dW, "dW", dev, X.dtype, B * V * D), p, ws.numel(), stream),
           "tokens_logprobs_grad")
    return dX, dW
