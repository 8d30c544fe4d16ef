"""Operators on token tables: ctypes binding of ``include/flashtokens.h``.

Argument marshalling only, as in :mod:`.kmeans`: tensors must be contiguous CUDA
(HIP) tensors on the current device, work is enqueued on torch's current stream,
and every output may be passed in.  A table is ``[V, D]`` (one instance) or
``[B, V, D]``; tokens are int32, and a token outside ``[0, V)`` is none.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

import torch

from .kmeans import _DTYPE, ERR_UNSUPPORTED, KMeansError, _check, _need, _ptr, _stream, lib

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


def _dt(t: torch.Tensor, name: str) -> int:
    try:
        return _DTYPE[t.dtype]
    except KeyError:
        raise TypeError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}") from None


def _rows(t: torch.Tensor, name: str) -> torch.Tensor:
    """[B, rows, D], or [rows, D] as one instance."""
    if t.dim() not in (2, 3):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, want [rows, D] or [B, rows, D]")
    return t if t.dim() == 3 else t.unsqueeze(0)


def _out(t: Optional[torch.Tensor], name: str, shape: Tuple[int, ...], dtype, device) -> torch.Tensor:
    if t is None:
        return torch.empty(shape, dtype=dtype, device=device)
    n = 1
    for s in shape:
        n *= s
    _need(t, name, dtype, n)
    return t


def _workspace(ws: Optional[torch.Tensor], need: int, where: str, device) -> torch.Tensor:
    if need == 0:
        raise KMeansError(ERR_UNSUPPORTED, where)
    if ws is None or ws.numel() < need:
        ws = torch.empty(need, dtype=torch.uint8, device=device)
    _need(ws, "ws", torch.uint8)
    return ws


def tokens_embed(table: torch.Tensor, idx: torch.Tensor, scale: float = 1.0,
                 out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """scale * table[idx], ``[B, M, D]``; zero rows where there is no token (see
    ``tokens_embed`` in the header)."""
    dt = _dt(table, "table")
    W = _rows(table, "table")
    B, V, D = W.shape
    _need(W, "table")
    _need(idx, "idx", torch.int32)
    M = idx.numel() // B if B else 0
    if idx.dim() == 2 and idx.shape[0] != B or idx.dim() not in (1, 2) or M * B != idx.numel():
        raise ValueError(f"idx has shape {tuple(idx.shape)}, want [B, M] with B = {B}")
    out = _out(out, "out", (B, M, D), table.dtype, table.device)
    _check(lib.tokens_embed(_ptr(W), dt, _ptr(idx), B, M, V, D, float(scale), _ptr(out), _stream()),
           "tokens_embed")
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
    G = _rows(grad, "grad")
    B, M, D = G.shape
    _need(G, "grad")
    _need(idx, "idx", torch.int32, B * M)
    if accumulate and out is None:
        raise ValueError("accumulate adds to out: pass it in")
    if out is not None and out.dtype not in (grad.dtype, torch.float32):
        raise TypeError(f"out must be {grad.dtype} or float32, got {out.dtype}")
    out = _out(out, "out", (B, V, D), grad.dtype if out is None else out.dtype, grad.device)
    ws = _workspace(ws, embed_grad_workspace_bytes(B, M, V, D, grad.dtype), "tokens_embed_grad",
                    grad.device)
    _check(lib.tokens_embed_grad(_ptr(G), dt, _ptr(idx), B, M, V, D, float(scale), int(accumulate),
                                 _ptr(out), _DTYPE[out.dtype], _ptr(ws), ws.numel(), _stream()),
           "tokens_embed_grad")
    return out


def _scored(X: torch.Tensor, W: torch.Tensor, bias: Optional[torch.Tensor]):
    X, W = _rows(X, "X"), _rows(W, "W")
    if X.shape[0] != W.shape[0] or X.shape[2] != W.shape[2]:
        raise ValueError(f"shapes X{tuple(X.shape)} W{tuple(W.shape)}: want [B,M,D] and [B,V,D]")
    dt = _dt(X, "X")
    if X.dtype != W.dtype:
        raise TypeError("rows and table must share a dtype")
    _need(X, "X")
    _need(W, "W")
    if bias is not None:
        _need(bias, "bias", torch.float32, W.shape[0] * W.shape[1])
    return X, W, dt


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
    X, W, dt = _scored(X, W, bias)
    B, M, D = X.shape
    V, dev, k = W.shape[1], X.device, int(k)
    if target is not None:
        _need(target, "target", torch.int32, B * M)
        logprob = _out(logprob, "logprob", (B, M), torch.float32, dev)
    elif logprob is not None:
        raise ValueError("logprob needs a target")
    entropy = _out(entropy, "entropy", (B, M), torch.float32, dev)
    lse = _out(lse, "lse", (B, M), torch.float32, dev)
    if k:
        top_idx = _out(top_idx, "top_idx", (B, M, k), torch.int32, dev)
        top_logprob = _out(top_logprob, "top_logprob", (B, M, k), torch.float32, dev)
    elif top_idx is not None or top_logprob is not None:
        raise ValueError("top_idx and top_logprob need k > 0")
    ws = _workspace(ws, logprobs_workspace_bytes(B, M, V, D, k, X.dtype), "tokens_logprobs", dev)
    _check(lib.tokens_logprobs(_ptr(X), _ptr(W), dt, _ptr(bias), _ptr(target), B, M, V, D, float(scale),
                               k, _ptr(logprob), _ptr(entropy), _ptr(lse), _ptr(top_idx),
                               _ptr(top_logprob), _ptr(ws), ws.numel(), _stream()), "tokens_logprobs")
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
    X, W, dt = _scored(X, W, bias)
    B, M, D = X.shape
    V, dev = W.shape[1], X.device
    _need(target, "target", torch.int32, B * M)
    _need(lse, "lse", torch.float32, B * M)
    _need(grad_logprob, "grad_logprob", torch.float32, B * M)
    if grad_entropy is not None:
        if entropy is None:
            raise ValueError("grad_entropy needs the entropy of the forward pass")
        _need(grad_entropy, "grad_entropy", torch.float32, B * M)
        _need(entropy, "entropy", torch.float32, B * M)
    else:
        entropy = None
    dX = _out(dX, "dX", (B, M, D), X.dtype, dev)
    dW = _out(dW, "dW", (B, V, D), W.dtype, dev)
    ws = _workspace(ws, logprobs_grad_workspace_bytes(B, M, V, D, X.dtype), "tokens_logprobs_grad", dev)
    _check(lib.tokens_logprobs_grad(_ptr(X), _ptr(W), dt, _ptr(bias), _ptr(target), _ptr(lse),
                                    _ptr(entropy), _ptr(grad_logprob), _ptr(grad_entropy), B, M, V, D,
                                    float(scale), _ptr(dX), _ptr(dW), _ptr(ws), ws.numel(), _stream()),
           "tokens_logprobs_grad")
    return dX, dW
