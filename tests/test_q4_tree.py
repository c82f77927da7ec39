"""Trees of drafts, kept rows and positions with axes without a GPU: refusals before any
launch."""
import ctypes as C

import pytest

from paper_2606_10944_amd import _lib
from test_q4 import BAD_CACHES, FAKE, ODD, cache

EINVAL, EDTYPE, EWORKSPACE = _lib.THIN_EINVAL, _lib.THIN_EDTYPE, _lib.THIN_EWORKSPACE
BYTE = C.c_void_p(0x10001)
FOUR = C.c_void_p(0x10004)


def axes(**kw):
    a = dict(X=FAKE, xs=None, Hx=4, XO=FAKE, xos=None, Y=FAKE, ys=None, Hy=2, YO=FAKE, yos=None,
             dtype=1, B=2, T=3, d=64, rot=32, layout=0, pos=FAKE, axes=3, axis=FAKE, turns=FAKE,
             amp=1.0, inverse=0)
    a.update(kw)
    return _lib.lib().thin_rotary_axes(*a.values(), None)


@pytest.mark.parametrize("kw,want", [
    (dict(axes=0), EINVAL), (dict(axes=5), EINVAL), (dict(axis=None), EINVAL),
    (dict(axis=BYTE), EINVAL), (dict(pos=None), EINVAL), (dict(X=None), EINVAL),
    (dict(X=ODD), EINVAL), (dict(dtype=2), EDTYPE), (dict(rot=24), EINVAL),
    (dict(rot=80), EINVAL), (dict(d=96), EINVAL), (dict(layout=2), EINVAL),
    (dict(turns=None), EINVAL), (dict(amp=float("nan")), EINVAL), (dict(B=0), EINVAL),
    (dict(T=0), EINVAL), (dict(B=1 << 27, T=2), EINVAL), (dict(Y=None), EINVAL)])
def test_rotary_axes_refusals(kw, want):
    assert axes(**kw) == want


def tree(**kw):
    a = dict(parents=FAKE, at=FAKE, B=2, T=10, seen=C.c_void_p(0x20000), pos=C.c_void_p(0x30000))
    a.update(kw)
    return _lib.lib().thin_q4_tree(*a.values(), None)


@pytest.mark.parametrize("kw", [
    dict(parents=None), dict(parents=BYTE), dict(at=None), dict(B=0), dict(B=65536), dict(T=0),
    dict(T=1025), dict(seen=None), dict(seen=FOUR), dict(pos=None), dict(pos=BYTE), dict(seen=FAKE),
    dict(pos=FAKE), dict(at=C.c_void_p(0x30000)), dict(pos=C.c_void_p(0x20000))])
def test_tree_refusals(kw):
    assert tree(**kw) == EINVAL


def attend(c=None, **kw):
    a = dict(Q=FAKE, qs=None, Hq=4, dtype=1, T=10, at=FAKE, count=None, seen=FAKE, O=FAKE, os=None,
             ws=FAKE, wn=1 << 40)
    a.update(kw)
    return _lib.lib().thin_q4_tree_attention(c if c is not None else cache(), *a.values(), None)


@pytest.mark.parametrize("kw,want", [
    (dict(Q=None), EINVAL), (dict(Q=ODD), EINVAL), (dict(Hq=3), EINVAL), (dict(Hq=0), EINVAL),
    (dict(dtype=7), EDTYPE), (dict(T=0), EINVAL), (dict(T=1025), EINVAL), (dict(at=None), EINVAL),
    (dict(count=BYTE), EINVAL), (dict(seen=None), EINVAL), (dict(seen=FOUR), EINVAL),
    (dict(O=None), EINVAL), (dict(O=ODD), EINVAL)])
def test_tree_attention_refusals(kw, want):
    assert attend(**kw) == want


def test_tree_attention_needs_the_plan_s_workspace():
    n = C.c_size_t(0)
    assert _lib.lib().thin_q4_attention_plan(2, 2, 4, 20000, 64, 10, 0, C.byref(n)) == 0
    big = cache(n_max=20000)
    assert n.value > 0
    assert attend(big, ws=None) == EWORKSPACE
    assert attend(big, wn=16) == EWORKSPACE
    assert attend(big, ws=ODD) == EWORKSPACE


def keep(c=None, **kw):
    a = dict(at=FAKE, path=C.c_void_p(0x20000), P=5, end=C.c_void_p(0x30000))
    a.update(kw)
    return _lib.lib().thin_q4_keep(c if c is not None else cache(), *a.values(), None)


@pytest.mark.parametrize("kw", [
    dict(at=None), dict(at=BYTE), dict(path=None), dict(path=BYTE), dict(P=0), dict(P=1025),
    dict(end=None), dict(end=BYTE), dict(end=FAKE)])
def test_keep_refusals(kw):
    assert keep(**kw) == EINVAL


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_bad_caches_are_refused(bad):
    assert attend(cache(**bad)) == EINVAL
    assert keep(cache(**bad)) == EINVAL
