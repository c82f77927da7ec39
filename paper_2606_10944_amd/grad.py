"""The gradient of coreset attention: binding of thin_attention_backward of include/thin.h
(argument marshalling only), and coreset attention as a function that autograd records."""
from __future__ import annotations

import ctypes as C
from functools import lru_cache
from typing import Optional

import torch

from ._lib import THIN_EDTYPE, THIN_EINVAL, ThinError, _check, _shape4, lib, thin_attention
from .q4 import _dtype, _empty, _on, _where, _workspace


@lru_cache(maxsize=4096)
def _bytes(dtype: int, B: int, H: int, n_q: int, n: int, d: int, n_out: int) -> int:
    need = C.c_size_t(0)
    _check(lib().thin_attention_backward_plan(dtype, B, H, n_q, n, d, n_out, C.byref(need)),
           "thin_attention_backward_plan")
    return need.value


def _gradient(t: Optional[torch.Tensor], shape, dtype: torch.dtype, dev: int, stream, name: str):
    if t is None:
        return _empty(shape, dtype, dev, stream)
    if t.shape != shape or t.dtype != dtype or not t.is_contiguous():
        raise ThinError(THIN_EINVAL, f"{name} must be contiguous {dtype} {list(shape)}")
    return t


def thin_attention_backward(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, idx: torch.Tensor,
                            dO: torch.Tensor, *, logw: Optional[torch.Tensor] = None,
                            dQ: Optional[torch.Tensor] = None, dK: Optional[torch.Tensor] = None,
                            dV: Optional[torch.Tensor] = None,
                            dlogw: Optional[torch.Tensor] = None, need_logw: bool = False,
                            workspace: Optional[torch.Tensor] = None, stream=None):
    """The gradients (dQ, dK, dV) of thin_attention(Q, K, V, idx, logw=logw) from dO, that of its
    output (float32 or bf16), with dlogw float32 [B,H,n_out] behind them when need_logw=True (or
    dlogw is given).  dK and dV are [B,H,n,d], zeros in the rows that idx does not list.  The
    forward's output is not needed."""
    dev, st = _where(stream)
    B, H, n_q, d = _shape4(Q, "Q")
    Bk, Hk, n, dk = _shape4(K, "K")
    if (Bk, Hk, dk) != (B, H, d) or _shape4(V, "V") != (B, H, n, d):
        raise ThinError(THIN_EINVAL, "Q/K/V shapes disagree")
    if K.dtype != Q.dtype or V.dtype != Q.dtype:
        raise ThinError(THIN_EDTYPE, "Q, K, V must share a dtype")
    if _shape4(dO, "dO") != (B, H, n_q, d):
        raise ThinError(THIN_EINVAL, "dO must match Q")
    if idx.dtype != torch.int32 or idx.dim() != 3 or idx.shape[:2] != (B, H) \
            or not idx.is_contiguous():
        raise ThinError(THIN_EINVAL, "idx must be contiguous int32 [B,H,n_out]")
    n_out = idx.shape[2]
    w = None
    if logw is not None:
        if logw.dtype != torch.float32 or logw.shape != (B, H, n_out) or not logw.is_contiguous():
            raise ThinError(THIN_EINVAL, "logw must be contiguous float32 [B,H,n_out]")
        w = _on(logw, dev, "logw")
    code, out_code = _dtype(Q, "Q"), _dtype(dO, "dO")
    ins = [_on(t, dev, name) for t, name in ((Q, "Q"), (K, "K"), (V, "V"), (idx, "idx"),
                                             (dO, "dO"))]
    need = _bytes(code, B, H, n_q, n, d, n_out)
    need_logw = need_logw or dlogw is not None
    dQ = _gradient(dQ, Q.shape, Q.dtype, dev, stream, "dQ")
    dK = _gradient(dK, K.shape, K.dtype, dev, stream, "dK")
    dV = _gradient(dV, V.shape, V.dtype, dev, stream, "dV")
    if need_logw:
        dlogw = _gradient(dlogw, idx.shape, torch.float32, dev, stream, "dlogw")
    ws, wp, wn = _workspace(workspace, need, dev, stream)
    _check(lib().thin_attention_backward(
        ins[0], ins[1], ins[2], code, B, H, n_q, n, d, ins[3], w, n_out, ins[4], out_code,
        _on(dQ, dev, "dQ"), _on(dK, dev, "dK"), _on(dV, dev, "dV"),
        _on(dlogw, dev, "dlogw") if need_logw else None, wp, wn, st), "thin_attention_backward")
    return (dQ, dK, dV, dlogw) if need_logw else (dQ, dK, dV)


class _CoresetAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, Q, K, V, idx, logw, out_dtype):
        ctx.save_for_backward(Q, K, V, idx, logw)
        return thin_attention(Q, K, V, idx, logw=logw, out_dtype=out_dtype)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dO):
        Q, K, V, idx, logw = ctx.saved_tensors
        with torch.cuda.device(Q.device):
            g = thin_attention_backward(Q, K, V, idx, dO.contiguous(), logw=logw,
                                        need_logw=ctx.needs_input_grad[4])
        return g[0], g[1], g[2], None, g[3] if ctx.needs_input_grad[4] else None, None


def coreset_attention(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, idx: torch.Tensor, *,
                      logw: Optional[torch.Tensor] = None,
                      out_dtype: torch.dtype = torch.float32) -> torch.Tensor:
    """thin_attention that autograd records, on the current stream: gradients reach Q, K, V
    (zeros in the rows that idx does not list) and logw by thin_attention_backward.  The choice
    of the rows, idx, has none.  Strided inputs are laid out contiguously first."""
    idx = idx.contiguous()
    if logw is not None:
        logw = logw.contiguous()
    return _CoresetAttention.apply(Q.contiguous(), K.contiguous(), V.contiguous(), idx, logw,
                                   out_dtype)
