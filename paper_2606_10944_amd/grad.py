"""The gradient of coreset attention: binding of thin_attention_backward of include/thin.h
(argument marshalling only), and coreset attention as a function that autograd records."""
from __future__ import annotations

import ctypes as C
from functools import lru_cache
from typing import Optional

import torch

from ._lib import THIN_EDTYPE, THIN_EINVAL, ThinError, _check, _shape4, lib, thin_attention
from .q4 import _dtype, _empty, _empty_like, _on, _where, _workspace


@lru_cache(maxsize=4096)
def _bytes(dtype: int, B: int, H: int, n_q: int, n: int, d: int, n_out: int) -> int:
    need = C.c_size_t(0)
    _check(lib().thin_attention_backward_plan(dtype, B, H, n_q, n, d, n_out, C.byref(need)),
           "thin_attention_backward_plan")
    return need.value


def _rows4(t: torch.Tensor, dev: int, name: str) -> int:
    """The address of contiguous rows [B,H,rows,d] on device `dev`."""
    if t.dim() != 4 or not t.is_contiguous():
        raise ThinError(THIN_EINVAL, f"{name} must be a contiguous [B,H,rows,d] tensor")
    return _on(t, dev, name)


def _gradient(t: torch.Tensor, like: torch.Tensor, dev: int, name: str) -> int:
    if t.shape != like.shape or t.dtype != like.dtype or not t.is_contiguous():
        raise ThinError(THIN_EINVAL, f"{name} must be contiguous {like.dtype} {list(like.shape)}")
    return _on(t, dev, name)


def thin_attention_backward(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, idx: torch.Tensor,
                            dO: torch.Tensor, *, logw: Optional[torch.Tensor] = None,
                            dQ: Optional[torch.Tensor] = None, dK: Optional[torch.Tensor] = None,
                            dV: Optional[torch.Tensor] = None,
                            dlogw: Optional[torch.Tensor] = None, need_logw: bool = False,
                            workspace: Optional[torch.Tensor] = None, stream=None):
    """The gradients (dQ, dK, dV) of thin_attention(Q, K, V, idx, logw=logw) from dO, that of its
    output (float32 or bf16), with dlogw float32 [B,H,n_out] behind them when need_logw=True (or
    dlogw is given).  Rows are contiguous and 16-byte aligned.  dK and dV are [B,H,n,d], zeros in
    the rows that idx does not list (entries outside [0, n) list the nearest row, as in the
    forward).  The forward's output is not needed."""
    dev, st = _where(stream)
    q, k, v, do = (_rows4(Q, dev, "Q"), _rows4(K, dev, "K"), _rows4(V, dev, "V"),
                   _rows4(dO, dev, "dO"))
    B, H, n_q, d = Q.shape
    n = K.shape[2]
    if K.shape != (B, H, n, d) or V.shape != K.shape:
        raise ThinError(THIN_EINVAL, "Q/K/V shapes disagree")
    dt = Q.dtype
    if K.dtype != dt or V.dtype != dt:
        raise ThinError(THIN_EDTYPE, "Q, K, V must share a dtype")
    if dO.shape != Q.shape:
        raise ThinError(THIN_EINVAL, "dO must match Q")
    n_out = idx.shape[2] if idx.dim() == 3 else 0
    if idx.dtype != torch.int32 or idx.shape != (B, H, n_out) or not idx.is_contiguous():
        raise ThinError(THIN_EINVAL, "idx must be contiguous int32 [B,H,n_out]")
    i = _on(idx, dev, "idx")
    w = None
    if logw is not None:
        if logw.dtype != torch.float32 or logw.shape != idx.shape or not logw.is_contiguous():
            raise ThinError(THIN_EINVAL, "logw must be contiguous float32 [B,H,n_out]")
        w = _on(logw, dev, "logw")
    code, out_code = _dtype(Q, "Q"), _dtype(dO, "dO")
    need = _bytes(code, B, H, n_q, n, d, n_out)
    if dQ is None:
        dQ = _empty_like(Q, dev, stream)
    if dK is None:
        dK = _empty_like(K, dev, stream)
    if dV is None:
        dV = _empty_like(V, dev, stream)
    g = (_gradient(dQ, Q, dev, "dQ"), _gradient(dK, K, dev, "dK"), _gradient(dV, V, dev, "dV"))
    dw = None
    if need_logw or dlogw is not None:
        if dlogw is None:
            dlogw = _empty(idx.shape, torch.float32, dev, stream)
        elif dlogw.dtype != torch.float32 or dlogw.shape != idx.shape \
                or not dlogw.is_contiguous():
            raise ThinError(THIN_EINVAL, "dlogw must be contiguous float32 [B,H,n_out]")
        dw = _on(dlogw, dev, "dlogw")
    ws, wp, wn = _workspace(workspace, need, dev, stream)
    rc = lib().thin_attention_backward(q, k, v, code, B, H, n_q, n, d, i, w, n_out, do, out_code,
                                       g[0], g[1], g[2], dw, wp, wn, st)
    if rc:
        _check(rc, "thin_attention_backward")
    return (dQ, dK, dV) if dw is None else (dQ, dK, dV, dlogw)


def _laid_out(t: torch.Tensor) -> torch.Tensor:
    """t, or a copy of it whose rows are contiguous and 16-byte aligned (a view into a flat buffer,
    or the gradient of a concatenation, may begin anywhere)."""
    t = t.contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone()


class _CoresetAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, Q, K, V, idx, logw, out_dtype):
        ctx.save_for_backward(Q, K, V, idx, logw)
        return thin_attention(Q, K, V, idx, logw=logw, out_dtype=out_dtype)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dO):
        Q, K, V, idx, logw = ctx.saved_tensors
        need_logw = ctx.needs_input_grad[4]
        with torch.cuda.device(Q.device):
            g = thin_attention_backward(Q, K, V, idx, _laid_out(dO), logw=logw,
                                        need_logw=need_logw)
        return g[0], g[1], g[2], None, g[3] if need_logw else None, None


def coreset_attention(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, idx: torch.Tensor, *,
                      logw: Optional[torch.Tensor] = None,
                      out_dtype: torch.dtype = torch.float32) -> torch.Tensor:
    """thin_attention that autograd records, on the current stream: gradients reach Q, K, V
    (zeros in the rows that idx does not list) and logw by thin_attention_backward, once (the
    gradient of a gradient is refused).  The choice of the rows, idx, has none.  A step that is
    captured into a graph calls thin_attention and thin_attention_backward itself.  Strided inputs
    are laid out contiguously first, and so are rows that are not 16-byte aligned.  Where a
    gradient is asked for, sizes that thin_attention_backward does not take are refused here."""
    dev, _ = _where(None)
    for t, name in ((Q, "Q"), (K, "K"), (V, "V"), (idx, "idx"), (logw, "logw")):
        if t is not None:
            _on(t, dev, name)
    code = _dtype(Q, "Q")
    recorded = torch.is_grad_enabled() and any(
        t is not None and t.requires_grad for t in (Q, K, V, logw))
    Q, K, V, idx = _laid_out(Q), _laid_out(K), _laid_out(V), idx.contiguous()
    if recorded:
        B, H, n_q, d = _shape4(Q, "Q")
        _bytes(code, B, H, n_q, _shape4(K, "K")[2], d, idx.shape[2] if idx.dim() == 3 else 0)
    return _CoresetAttention.apply(Q, K, V, idx, None if logw is None else logw.contiguous(),
                                   out_dtype)
