"""Rotary positions and the key/value cache held in 4 bits: binding of thin_rotary
and the thin_q4_* calls of include/thin.h (argument marshalling only).

Tensors and the given stream live on the current device; rows are [B, heads,
T, d] tensors of any strides with contiguous channels, 16-byte aligned.  No call
is recorded by autograd, whatever its inputs require: outputs are detached.  The
gradient of a turn is thin_rotary(..., inverse=True) of the gradient.
"""
from __future__ import annotations

import ctypes as C
from functools import lru_cache
from typing import Optional, Tuple

import torch

from ._lib import (THIN_BF16, THIN_EDTYPE, THIN_EINVAL, THIN_FP32, Q4CacheStruct, ThinError, _check,
                   lib)

BLOCK = 64  # THIN_Q4_BLOCK
MAX_DRAFTS = 1024  # THIN_Q4_MAX_DRAFTS
LAYOUT = {"half": 0, "interleaved": 1}
SCALING = {"none": 0, "linear": 1, "base": 2, "bands": 3}

_DTYPE = {torch.float32: THIN_FP32, torch.bfloat16: THIN_BF16}
_Strides = C.c_int64 * 3


_get_device = torch._C._cuda_getDevice
_raw_stream = torch._C._cuda_getCurrentRawStream


def _where(stream):
    """(device index, raw stream) that a call runs on: a stream of the current device."""
    dev = _get_device()
    if stream is None:
        return dev, _raw_stream(dev)
    if stream.device.index != dev:
        raise ThinError(THIN_EINVAL, f"the stream is on {stream.device}, the current device is "
                                     f"cuda:{dev}")
    return dev, stream.cuda_stream


def _empty(shape, dtype: torch.dtype, dev: int, stream) -> torch.Tensor:
    """Memory of the stream that the call runs on: the allocator hands memory out
    in the order of one stream, so what another stream uses comes from its own."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=dev)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=dev)


def _empty_like(t: torch.Tensor, dev: int, stream) -> torch.Tensor:
    """Contiguous memory for t's shape (half the host time of _empty)."""
    if stream is None and t.is_contiguous():
        return torch.empty_like(t)
    return _empty(t.shape, t.dtype, dev, stream)


def _dtype(t: torch.Tensor, name: str) -> int:
    code = _DTYPE.get(t.dtype)
    if code is None:
        raise ThinError(THIN_EDTYPE, f"{name}: {t.dtype}")
    return code


def _on(t: torch.Tensor, dev: int, name: str) -> int:
    """The tensor's address; it must live on device `dev`."""
    if t.get_device() != dev:
        raise ThinError(THIN_EINVAL, f"{name} is on {t.device}, the call on cuda:{dev}")
    return t.data_ptr()


def _rows(t: torch.Tensor, dev: int, name: str):
    """(address, strides or None if contiguous) of rows [B, heads, T, d]."""
    if t.dim() != 4:
        raise ThinError(THIN_EINVAL, f"{name} must be [B,heads,T,d]")
    p = _on(t, dev, name)
    if t.is_contiguous():
        return p, None
    s = t.stride()
    if s[3] != 1:
        raise ThinError(THIN_EINVAL, f"{name}: channels must be contiguous")
    return p, _Strides(s[0], s[1], s[2])


def _addressable(t: torch.Tensor, strides, name: str, output: bool = False) -> None:
    """Refuses rows that the library would for their alignment or strides."""
    word = 16 // t.element_size()
    bad = t.data_ptr() % 16 != 0
    if strides is not None:
        bad = bad or any(n > 1 and (s % word != 0 or (output and s == 0))
                         for n, s in zip(t.shape, strides))
    if bad:
        raise ThinError(THIN_EINVAL, f"{name}: rows must be 16-byte aligned"
                                     f"{' and apart' if output else ''}")


def _ints(t: Optional[torch.Tensor], shape, dev: int, name: str):
    if t is None:
        return None
    if t.dtype != torch.int32 or t.shape != shape or not t.is_contiguous():
        raise ThinError(THIN_EINVAL, f"{name} must be contiguous int32 {list(shape)}")
    return _on(t, dev, name)


def _workspace(ws: Optional[torch.Tensor], need: int, dev: int, stream):
    """(tensor to keep, address, bytes) of a call's workspace."""
    if ws is None:
        if need == 0:
            return None, None, 0
        ws = _empty(need, torch.uint8, dev, stream)
    elif not ws.is_contiguous():
        raise ThinError(THIN_EINVAL, "workspace must be contiguous")
    return ws, _on(ws, dev, "workspace"), ws.numel() * ws.element_size()


def thin_rotary_turns(rot: int, *, base: float = 10000.0, scaling: str = "none",
                      factor: float = 1.0, length: float = 0.0, slow: float = 1.0,
                      fast: float = 32.0) -> Tuple[torch.Tensor, float]:
    """(turns, amp) of thin_rotary for a head whose first `rot` channels turn:
    base^(-2i/rot) / 2 pi turns per position (a float64 CPU tensor [rot/2]),
    stretched for contexts `factor` times as long as `length` by one of the rules
    "linear", "base" and "bands" (thin_rotary_turns in include/thin.h).  amp is
    0.1 ln(factor) + 1 with "bands", else 1; models trained with the bands but
    without that factor pass amp=1."""
    if scaling not in SCALING:
        raise ThinError(THIN_EINVAL, f"unknown scaling {scaling!r}")
    turns = torch.empty(max(int(rot) // 2, 1), dtype=torch.float64)
    amp = C.c_double(0.0)
    _check(lib().thin_rotary_turns(rot, base, SCALING[scaling], factor, length, slow, fast,
                                   turns.data_ptr(), C.byref(amp)), "thin_rotary_turns")
    return turns, amp.value


def thin_rotary(X: torch.Tensor, pos: torch.Tensor, turns: torch.Tensor, *,
                Y: Optional[torch.Tensor] = None, layout: str = "half", amp: float = 1.0,
                inverse: bool = False, out: Optional[torch.Tensor] = None,
                out_Y: Optional[torch.Tensor] = None, stream=None):
    """Rows X [B,heads,T,d], and Y [B,heads',T,d] in the same launch, turned by
    their positions: pos int32 [B,T], or [B], the first row's.  turns float64
    [rot/2] on the device.  inverse=True turns back: of an output's gradient, the
    gradient of the rows (autograd does not record the call).
    out / out_Y may be X / Y themselves.  Returns out, or (out, out_Y) with Y."""
    return _rotary(X, pos, turns, None, Y, layout, amp, inverse, out, out_Y, stream)


def thin_rotary_axes(X: torch.Tensor, pos: torch.Tensor, turns: torch.Tensor, axis: torch.Tensor,
                     *, Y: Optional[torch.Tensor] = None, layout: str = "half", amp: float = 1.0,
                     inverse: bool = False, out: Optional[torch.Tensor] = None,
                     out_Y: Optional[torch.Tensor] = None, stream=None):
    """thin_rotary with several positions per token (time, height, width): pos
    int32 [B,T,axes], up to 4 axes, and axis int32 [rot/2] on the device, the axis
    of every pair of channels."""
    if pos.dim() != 3:
        raise ThinError(THIN_EINVAL, "pos must be int32 [B,T,axes]")
    if axis.dim() != 1 or axis.shape != turns.shape:
        raise ThinError(THIN_EINVAL, "axis must be int32 [rot/2], as turns")
    return _rotary(X, pos, turns, axis, Y, layout, amp, inverse, out, out_Y, stream)


def _rotary(X, pos, turns, axis, Y, layout, amp, inverse, out, out_Y, stream):
    dev, st = _where(stream)
    lay = LAYOUT.get(layout)
    if lay is None:
        raise ThinError(THIN_EINVAL, f"unknown layout {layout!r}")
    x, xs = _rows(X, dev, "X")
    shape = X.shape
    B, H, T, d = shape
    if turns.dtype != torch.float64 or turns.dim() != 1 or not turns.is_contiguous():
        raise ThinError(THIN_EINVAL, "turns must be contiguous float64 [rot/2]")
    if axis is None:
        per_token = pos.dim() == 2
        p = _ints(pos, (B, T) if per_token else (B,), dev, "pos")
    else:
        axes = pos.shape[2]
        p = _ints(pos, (B, T, axes), dev, "pos")
    if out is None:
        out = _empty_like(X, dev, stream)
        o, os_ = out.data_ptr(), None
    else:
        if out.shape != shape or out.dtype != X.dtype:
            raise ThinError(THIN_EINVAL, "out must match X")
        o, os_ = _rows(out, dev, "out")
    y = ys = oy = oys = None
    Hy = 0
    if Y is not None:
        y, ys = _rows(Y, dev, "Y")
        Hy = Y.shape[1]
        if Y.shape != (B, Hy, T, d):
            raise ThinError(THIN_EINVAL, "Y must be [B,heads,T,d] with X's B, T and d")
        if Y.dtype != X.dtype:
            raise ThinError(THIN_EDTYPE, "X and Y must share a dtype")
        if out_Y is None:
            out_Y = _empty_like(Y, dev, stream)
            oy = out_Y.data_ptr()
        else:
            if out_Y.shape != Y.shape or out_Y.dtype != Y.dtype:
                raise ThinError(THIN_EINVAL, "out_Y must match Y")
            oy, oys = _rows(out_Y, dev, "out_Y")
    elif out_Y is not None:
        raise ThinError(THIN_EINVAL, "out_Y without Y")
    if axis is None:
        rc = lib().thin_rotary(x, xs, H, o, os_, y, ys, Hy, oy, oys, _dtype(X, "X"), B, T, d,
                               2 * turns.shape[0], lay, p, per_token, _on(turns, dev, "turns"),
                               amp, inverse, st)
    else:
        rc = lib().thin_rotary_axes(x, xs, H, o, os_, y, ys, Hy, oy, oys, _dtype(X, "X"), B, T, d,
                                    2 * turns.shape[0], lay, p, axes,
                                    _ints(axis, axis.shape, dev, "axis"),
                                    _on(turns, dev, "turns"), amp, inverse, st)
    if rc:
        _check(rc, "thin_rotary" if axis is None else "thin_rotary_axes")
    return out if Y is None else (out, out_Y)


class Q4Cache:
    """Key/value rows of B sequences and H key heads, up to n_max each, held in 4
    bits (thin_q4_cache_t): codes and scales of keys and values, and the bounds of
    the keys of every 64 rows.  The buffers are plain tensors of the object.

    ``step`` is one decoding step or one prompt (or a chunk of it): new queries,
    keys and values, turned by their positions if `turns` is given, the rows
    stored, and attention over the cache or over the blocks selected from it.
    ``draft`` is a step of a tree of drafted tokens, ``keep`` takes the accepted ones."""

    def __init__(self, B: int, H: int, n_max: int, d: int, *, device="cuda"):
        nb = (n_max + BLOCK - 1) // BLOCK
        u8 = dict(dtype=torch.uint8, device=device)
        self._set(torch.empty((B, H, n_max, d // 2), **u8),
                  torch.empty((B, H, n_max, d // 32), **u8),
                  torch.empty((B, H, n_max, d // 2), **u8),
                  torch.empty((B, H, n_max, d // 32), **u8),
                  torch.empty((B, H, nb, 2, d), dtype=torch.bfloat16, device=device))

    @classmethod
    def over(cls, k_codes: torch.Tensor, k_scales: torch.Tensor, v_codes: torch.Tensor,
             v_scales: torch.Tensor, bounds: torch.Tensor) -> "Q4Cache":
        """A cache over existing buffers of these shapes."""
        self = cls.__new__(cls)
        self._set(k_codes, k_scales, v_codes, v_scales, bounds)
        return self

    def _set(self, k_codes, k_scales, v_codes, v_scales, bounds):
        if k_codes.dim() != 4:
            raise ThinError(THIN_EINVAL, "k_codes must be [B,H,n_max,d/2]")
        B, H, n, half = k_codes.shape
        d = 2 * half
        if d not in (32, 64, 128):
            raise ThinError(THIN_EINVAL, "d must be 32, 64 or 128")
        want = {"k_codes": (B, H, n, half), "k_scales": (B, H, n, d // 32),
                "v_codes": (B, H, n, half), "v_scales": (B, H, n, d // 32),
                "bounds": (B, H, (n + BLOCK - 1) // BLOCK, 2, d)}
        self.k_codes, self.k_scales, self.v_codes, self.v_scales, self.bounds = \
            k_codes, k_scales, v_codes, v_scales, bounds
        for name, shape in want.items():
            t = getattr(self, name)
            dt = torch.bfloat16 if name == "bounds" else torch.uint8
            if t.shape != shape or t.dtype != dt or not t.is_contiguous() \
                    or t.device != k_codes.device:
                raise ThinError(THIN_EINVAL, f"{name} must be contiguous {dt} {list(shape)}")
        self.B, self.H, self.n_max, self.d = B, H, n, d
        self.device_index = k_codes.get_device()
        self.struct = Q4CacheStruct(*[getattr(self, k).data_ptr() for k in want], B, H, n, d)
        self._ref = C.byref(self.struct)

    def _at(self, dev: int):
        if self.device_index != dev:
            raise ThinError(THIN_EINVAL, f"the cache is on {self.k_codes.device}, the call on "
                                         f"cuda:{dev}")
        return self._ref

    def step(self, Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, at: torch.Tensor, *,
             count: Optional[torch.Tensor] = None, turns: Optional[torch.Tensor] = None,
             layout: str = "half", amp: float = 1.0, n_sel: int = 0, n_sinks: int = 1,
             n_window: int = 2, O: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Outputs O [B,q_heads,T,d] of T new tokens per sequence at positions
        at[b] + t: queries Q [B,q_heads,T,d], rows K, V [B,H,T,d].  With n_sel they
        attend to n_sel blocks of 64 rows (thin_q4_select), else to every row.  A step
        that is refused has stored nothing."""
        self._check_step(Q, n_sel, n_sinks, n_window, O, _where(stream)[0])
        if turns is not None:
            Q, K = thin_rotary(Q, at, turns, Y=K, layout=layout, amp=amp, stream=stream)
        thin_q4_store(K, V, self, at, count=count, stream=stream)
        blocks = None
        if n_sel:
            blocks = thin_q4_select(Q, self, at, n_sel, n_sinks=n_sinks, n_window=n_window,
                                    count=count, stream=stream)
        return thin_q4_attention(Q, self, at, count=count, blocks=blocks, O=O, stream=stream)

    def draft(self, Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, at: torch.Tensor,
              parents: Optional[torch.Tensor] = None, *, count: Optional[torch.Tensor] = None,
              turns: Optional[torch.Tensor] = None, layout: str = "half", amp: float = 1.0,
              tree=None, pos: Optional[torch.Tensor] = None, axis: Optional[torch.Tensor] = None,
              O: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Outputs O [B,q_heads,T,d] of a tree of T drafted tokens behind the first at[b] rows:
        rows K, V [B,H,T,d] are stored at at[b] + t, turned (with `turns`) by the drafts'
        positions in the tree, and a draft attends to the rows before at[b], its ancestors and
        itself.  parents int32 [B,T] (thin_q4_tree).  Layers of one step share a tree:
        tree=(seen, pos) as thin_q4_tree gave them is taken in place of parents.
        Positions of their own: pos int32 [B,T], or [B,T,axes] with the pairs' `axis`
        (thin_rotary_axes).  keep() then takes the accepted rows.  A call that is refused has
        stored nothing."""
        self._check_step(Q, 0, 0, 1, O, _where(stream)[0])
        B, T = self.B, Q.shape[2]
        if T > MAX_DRAFTS:
            raise ThinError(THIN_EINVAL, f"at most {MAX_DRAFTS} drafts")
        if tree is None:
            if parents is None or parents.shape != (B, T):
                raise ThinError(THIN_EINVAL, "parents must be int32 [B,T]")
            tree = thin_q4_tree(parents, at, stream=stream)
        if K.dim() != 4 or K.shape[2] != T:
            raise ThinError(THIN_EINVAL, "K and V must have a row for every draft")
        seen = tree[0]
        _masks(seen, B, T, _where(stream)[0])
        if turns is not None:
            where = tree[1] if pos is None else pos
            if axis is not None:
                Q, K = thin_rotary_axes(Q, where, turns, axis, Y=K, layout=layout, amp=amp,
                                        stream=stream)
            else:
                if where.shape != (B, T):
                    raise ThinError(THIN_EINVAL, "pos must be int32 [B,T]")
                Q, K = thin_rotary(Q, where, turns, Y=K, layout=layout, amp=amp, stream=stream)
        elif pos is not None or axis is not None:
            raise ThinError(THIN_EINVAL, "pos and axis need turns")
        thin_q4_store(K, V, self, at, count=count, stream=stream)
        return thin_q4_tree_attention(Q, self, at, seen, count=count, O=O, stream=stream)

    def keep(self, at: torch.Tensor, path: torch.Tensor, *, end: Optional[torch.Tensor] = None,
             stream=None) -> torch.Tensor:
        """thin_q4_keep over this cache."""
        return thin_q4_keep(self, at, path, end=end, stream=stream)

    def _check_step(self, Q, n_sel, n_sinks, n_window, O, dev: int) -> None:
        """Refuses what the selection or attention of a step would, before its rows are
        stored."""
        self._at(dev)
        _, qs, Hq, T = _queries(Q, self, dev)
        _dtype(Q, "Q")
        _addressable(Q, qs, "Q")
        if n_sel and not (0 <= n_sinks and 1 <= n_window and n_sinks + n_window <= n_sel <= 32768):
            raise ThinError(THIN_EINVAL, "n_sinks >= 0, n_window >= 1 and n_sinks + n_window <= "
                                         "n_sel <= 32768")
        _attention_bytes(self.B, self.H, Hq, self.n_max, self.d, T, n_sel)
        if O is not None:
            _addressable(O, _output(O, Q, dev)[1], "O", output=True)


def thin_q4_store(K: torch.Tensor, V: torch.Tensor, cache: Q4Cache, at: torch.Tensor, *,
                  count: Optional[torch.Tensor] = None, stream=None) -> None:
    """Encode rows K, V [B,H,T,d] into rows at[b] + t of the cache (at int32 [B];
    tokens t >= count[b], int32 [B], are padding)."""
    dev, st = _where(stream)
    ref = cache._at(dev)
    k, ks = _rows(K, dev, "K")
    v, vs = _rows(V, dev, "V")
    B, H, T, d = K.shape
    if (B, H, d) != (cache.B, cache.H, cache.d) or V.shape != K.shape:
        raise ThinError(THIN_EINVAL, "K and V must be [B,H,T,d] of the cache's B, H and d")
    if V.dtype != K.dtype:
        raise ThinError(THIN_EDTYPE, "K and V must share a dtype")
    _check(lib().thin_q4_store(ref, k, ks, v, vs, _dtype(K, "K"), T,
                               _ints(at, (B,), dev, "at"), _ints(count, (B,), dev, "count"), st),
           "thin_q4_store")


def thin_q4_load(cache: Q4Cache, at: torch.Tensor, T: int, *,
                 dtype: torch.dtype = torch.bfloat16, K: Optional[torch.Tensor] = None,
                 V: Optional[torch.Tensor] = None, stream=None):
    """(K, V) [B,H,T,d]: the values that rows at[b] .. at[b] + T - 1 of the cache
    stand for, zeros outside the cache."""
    dev, st = _where(stream)
    ref = cache._at(dev)
    shape = (cache.B, cache.H, T, cache.d)
    if K is None:
        K = _empty(shape, dtype, dev, stream)
    if V is None:
        V = _empty_like(K, dev, stream)
    for t, name in ((K, "K"), (V, "V")):
        if t.shape != shape or not t.is_contiguous() or t.dtype != K.dtype:
            raise ThinError(THIN_EINVAL, f"{name} must be contiguous [B,H,T,d]")
    _check(lib().thin_q4_load(ref, T, _ints(at, (cache.B,), dev, "at"), _on(K, dev, "K"),
                              _on(V, dev, "V"), _dtype(K, "K"), st), "thin_q4_load")
    return K, V


@lru_cache(maxsize=4096)
def _select_bytes(B: int, H: int, n_max: int, T: int) -> int:
    n = C.c_size_t(0)
    _check(lib().thin_q4_select_plan(B, H, n_max, T, C.byref(n)), "thin_q4_select_plan")
    return n.value


@lru_cache(maxsize=4096)
def _attention_bytes(B: int, H: int, Hq: int, n_max: int, d: int, T: int, n_sel: int) -> int:
    n = C.c_size_t(0)
    _check(lib().thin_q4_attention_plan(B, H, Hq, n_max, d, T, n_sel, C.byref(n)),
           "thin_q4_attention_plan")
    return n.value


def _queries(Q: torch.Tensor, cache: Q4Cache, dev: int):
    q, qs = _rows(Q, dev, "Q")
    B, Hq, T, d = Q.shape
    if B != cache.B or d != cache.d or Hq < 1 or Hq % cache.H:
        raise ThinError(THIN_EINVAL, "Q must be [B,q_heads,T,d] of the cache's B and d, q_heads a "
                                     "multiple of its H")
    return q, qs, Hq, T


def _output(O: torch.Tensor, Q: torch.Tensor, dev: int):
    if O.shape != Q.shape or O.dtype != Q.dtype:
        raise ThinError(THIN_EINVAL, "O must match Q")
    return _rows(O, dev, "O")


def thin_q4_select(Q: torch.Tensor, cache: Q4Cache, at: torch.Tensor, n_sel: int, *,
                   n_sinks: int = 1, n_window: int = 2, count: Optional[torch.Tensor] = None,
                   blocks: Optional[torch.Tensor] = None,
                   workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """blocks [B,H,T,n_sel] int32: for every token and key head the first n_sinks
    and last n_window blocks of 64 rows up to the token's own, and those that its
    queries could score highest in, ascending, -1 behind."""
    dev, st = _where(stream)
    ref = cache._at(dev)
    q, qs, Hq, T = _queries(Q, cache, dev)
    B, H = cache.B, cache.H
    need = _select_bytes(B, H, cache.n_max, T)
    if blocks is None:
        if n_sel < 1:
            raise ThinError(THIN_EINVAL, "n_sel must be at least 1")
        blocks = _empty((B, H, T, n_sel), torch.int32, dev, stream)
    b = _ints(blocks, (B, H, T, n_sel), dev, "blocks")
    ws, wp, wn = _workspace(workspace, need, dev, stream)
    _check(lib().thin_q4_select(ref, q, qs, Hq, _dtype(Q, "Q"), T, _ints(at, (B,), dev, "at"),
                                _ints(count, (B,), dev, "count"), n_sel, n_sinks, n_window, b,
                                wp, wn, st), "thin_q4_select")
    return blocks


def thin_q4_attention(Q: torch.Tensor, cache: Q4Cache, at: torch.Tensor, *,
                      count: Optional[torch.Tensor] = None,
                      blocks: Optional[torch.Tensor] = None, O: Optional[torch.Tensor] = None,
                      workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Causal attention of queries Q [B,q_heads,T,d] at positions at[b] + t over the
    cached rows up to each, or over those in the token's listed blocks (int32
    [B,H,T,n_sel], thin_q4_select).  Padding (t >= count[b]) gives rows of zeros."""
    dev, st = _where(stream)
    ref = cache._at(dev)
    q, qs, Hq, T = _queries(Q, cache, dev)
    B, H = cache.B, cache.H
    n_sel, bp = 0, None
    if blocks is not None:
        if blocks.dim() != 4 or blocks.shape[3] < 1:
            raise ThinError(THIN_EINVAL, "blocks must be int32 [B,H,T,n_sel]")
        n_sel = blocks.shape[3]
        bp = _ints(blocks, (B, H, T, n_sel), dev, "blocks")
    need = _attention_bytes(B, H, Hq, cache.n_max, cache.d, T, n_sel)
    if O is None:
        O = _empty_like(Q, dev, stream)
        o, os_ = O.data_ptr(), None
    else:
        o, os_ = _output(O, Q, dev)
    ws, wp, wn = _workspace(workspace, need, dev, stream)
    _check(lib().thin_q4_attention(ref, q, qs, Hq, _dtype(Q, "Q"), T, _ints(at, (B,), dev, "at"),
                                   _ints(count, (B,), dev, "count"), bp, n_sel, o, os_, wp, wn,
                                   st), "thin_q4_attention")
    return O


def thin_q4_tree(parents: torch.Tensor, at: torch.Tensor, *, seen: Optional[torch.Tensor] = None,
                 pos: Optional[torch.Tensor] = None, stream=None):
    """(seen, pos) of trees of drafted tokens: parents int32 [B,T], every draft's parent (an
    earlier draft; negative: a root).  seen int64 [B,T,ceil(T/64)]: bit j % 64 of word j / 64
    is set if draft t attends to draft j, itself and its ancestors.  pos int32 [B,T]: at[b] +
    the draft's depth, the positions of thin_rotary."""
    dev, st = _where(stream)
    if parents.dim() != 2:
        raise ThinError(THIN_EINVAL, "parents must be int32 [B,T]")
    B, T = parents.shape
    p, a = _ints(parents, (B, T), dev, "parents"), _ints(at, (B,), dev, "at")
    if seen is None:
        seen = _empty((B, T, (T + 63) // 64), torch.int64, dev, stream)
    if pos is None:
        pos = _empty((B, T), torch.int32, dev, stream)
    _check(lib().thin_q4_tree(p, a, B, T, _masks(seen, B, T, dev), _ints(pos, (B, T), dev, "pos"),
                              st), "thin_q4_tree")
    return seen, pos


def _masks(seen: torch.Tensor, B: int, T: int, dev: int) -> int:
    if seen.dtype != torch.int64 or seen.shape != (B, T, (T + 63) // 64) \
            or not seen.is_contiguous():
        raise ThinError(THIN_EINVAL, "seen must be contiguous int64 [B,T,ceil(T/64)]")
    return _on(seen, dev, "seen")


def thin_q4_tree_attention(Q: torch.Tensor, cache: Q4Cache, at: torch.Tensor, seen: torch.Tensor,
                           *, count: Optional[torch.Tensor] = None,
                           O: Optional[torch.Tensor] = None,
                           workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Attention of drafts Q [B,q_heads,T,d], T <= 1024, whose rows are at[b] + t of the cache,
    over the rows before at[b] and the drafts of their masks seen int64 [B,T,ceil(T/64)]
    (thin_q4_tree, or any other).  Padding (t >= count[b]) and drafts that see nothing give
    rows of zeros."""
    dev, st = _where(stream)
    ref = cache._at(dev)
    q, qs, Hq, T = _queries(Q, cache, dev)
    B, H = cache.B, cache.H
    if T > MAX_DRAFTS:
        raise ThinError(THIN_EINVAL, f"at most {MAX_DRAFTS} drafts")
    need = _attention_bytes(B, H, Hq, cache.n_max, cache.d, T, 0)
    if O is None:
        O = _empty_like(Q, dev, stream)
        o, os_ = O.data_ptr(), None
    else:
        o, os_ = _output(O, Q, dev)
    ws, wp, wn = _workspace(workspace, need, dev, stream)
    _check(lib().thin_q4_tree_attention(ref, q, qs, Hq, _dtype(Q, "Q"), T,
                                        _ints(at, (B,), dev, "at"),
                                        _ints(count, (B,), dev, "count"),
                                        _masks(seen, B, T, dev), o, os_, wp, wn, st),
           "thin_q4_tree_attention")
    return O


def thin_q4_keep(cache: Q4Cache, at: torch.Tensor, path: torch.Tensor, *,
                 end: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Rows at[b] + path[b,i] of the cache become rows at[b] + i (path int32 [B,P], P <= 1024,
    an accepted path of drafts, the first negative entry behind its last; padding, drafts t >=
    count[b], is not for a path: its rows were never stored).  Returns end int32 [B], the rows
    that every sequence then has: the next call's `at`."""
    dev, st = _where(stream)
    ref = cache._at(dev)
    if path.dim() != 2:
        raise ThinError(THIN_EINVAL, "path must be int32 [B,P]")
    B, P = cache.B, path.shape[1]
    if end is None:
        end = _empty((B,), torch.int32, dev, stream)
    _check(lib().thin_q4_keep(ref, _ints(at, (B,), dev, "at"), _ints(path, (B, P), dev, "path"), P,
                              _ints(end, (B,), dev, "end"), st), "thin_q4_keep")
    return end
