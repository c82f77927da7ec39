"""Rotary positions and the 4-bit cache without a GPU: refusals before any launch,
the tables of turns, the workspaces, the reference's own encoding."""
import ctypes as C
import math

import pytest
import torch

import q4_reference as ref
from paper_2606_10944_amd import Q4Cache, _lib, q4, thin_rotary_turns
from paper_2606_10944_amd._lib import Q4CacheStruct

FAKE = C.c_void_p(0x10000)  # never dereferenced: every call below fails validation
ODD = C.c_void_p(0x10008)   # not 16-byte aligned
EINVAL, EDTYPE, EWORKSPACE = _lib.THIN_EINVAL, _lib.THIN_EDTYPE, _lib.THIN_EWORKSPACE


def cache(**kw):
    a = dict(k_codes=FAKE, k_scales=FAKE, v_codes=FAKE, v_scales=FAKE, bounds=FAKE, B=2, H=2,
             n_max=1000, d=64)
    a.update(kw)
    return C.byref(Q4CacheStruct(*[a[f] for f, _ in Q4CacheStruct._fields_]))


def strides(*s):
    return (C.c_int64 * 3)(*s)


def test_a_stream_of_another_device_is_refused(monkeypatch):
    class Stream:
        device = torch.device("cuda", 1)
        cuda_stream = 4096

    monkeypatch.setattr(q4, "_get_device", lambda: 0)
    with pytest.raises(_lib.ThinError, match="cuda:1"):
        q4._where(Stream)
    monkeypatch.setattr(q4, "_get_device", lambda: 1)
    assert q4._where(Stream) == (1, 4096)


def test_attention_takes_as_many_rows_as_a_grid_holds():
    plan, n = _lib.lib().thin_q4_attention_plan, C.c_size_t(0)
    for n_sel in (0, 4):
        for G in (1, 100, 128):
            assert plan(1, 2, 2 * G, 5000, 64, 1 << 20, n_sel, C.byref(n)) == 0
        assert plan(1, 2, 2 * 129, 5000, 64, 1 << 20, n_sel, C.byref(n)) == EINVAL
        assert plan(32, 32, 32, 5000, 64, 1 << 20, n_sel, C.byref(n)) == 0
        assert plan(32, 33, 33, 5000, 64, 1 << 20, n_sel, C.byref(n)) == EINVAL


BAD_CACHES = [dict(k_codes=None), dict(bounds=None), dict(v_scales=ODD), dict(B=0), dict(H=-1),
              dict(B=300, H=300), dict(n_max=0), dict(n_max=(1 << 21) + 1), dict(d=96),
              dict(B=1 << 40, H=1 << 40)]


def rotary(**kw):
    a = dict(X=FAKE, xs=None, Hx=4, XO=FAKE, xos=None, Y=FAKE, ys=None, Hy=2, YO=FAKE, yos=None,
             dtype=1, B=2, T=3, d=64, rot=32, layout=0, pos=FAKE, per=0, turns=FAKE, amp=1.0,
             inverse=0)
    a.update(kw)
    return _lib.lib().thin_rotary(*a.values(), None)


@pytest.mark.parametrize("kw,want", [
    (dict(X=None), EINVAL), (dict(XO=None), EINVAL), (dict(YO=None), EINVAL),
    (dict(Y=None), EINVAL), (dict(Y=None, Hy=0), EINVAL), (dict(X=ODD), EINVAL),
    (dict(YO=ODD), EINVAL), (dict(dtype=2), EDTYPE), (dict(d=96), EINVAL), (dict(rot=0), EINVAL),
    (dict(rot=8), EINVAL), (dict(rot=80), EINVAL), (dict(rot=24), EINVAL),
    (dict(layout=2), EINVAL), (dict(pos=None), EINVAL), (dict(turns=None), EINVAL),
    (dict(amp=math.nan), EINVAL), (dict(amp=math.inf), EINVAL), (dict(B=0), EINVAL),
    (dict(T=0), EINVAL), (dict(Hx=0), EINVAL), (dict(Hy=0), EINVAL), (dict(Hx=70000), EINVAL),
    (dict(B=1 << 20, T=1 << 20), EINVAL), (dict(B=1 << 62, T=4), EINVAL),
    (dict(xs=strides(768, 100, 64)), EINVAL), (dict(xos=strides(0, 192, 64)), EINVAL),
    (dict(yos=strides(384, 192, 0)), EINVAL), (dict(dtype=0, xs=strides(768, 192, 2)), EINVAL)])
def test_rotary_refusals(kw, want):
    assert rotary(**kw) == want


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_bad_caches_are_refused(bad):
    L = _lib.lib()
    c = cache(**bad)
    assert L.thin_q4_store(c, FAKE, None, FAKE, None, 1, 1, FAKE, None, None) == EINVAL
    assert L.thin_q4_load(c, 1, FAKE, FAKE, FAKE, 1, None) == EINVAL
    assert L.thin_q4_select(c, FAKE, None, 4, 1, 1, FAKE, None, 4, 1, 1, FAKE, FAKE, 1 << 40,
                            None) == EINVAL
    assert L.thin_q4_attention(c, FAKE, None, 4, 1, 1, FAKE, None, None, 0, FAKE, None, FAKE,
                               1 << 40, None) == EINVAL


def test_store_and_load_refusals():
    L = _lib.lib()

    def store(K=FAKE, ks=None, V=FAKE, vs=None, dtype=1, T=5, at=FAKE):
        return L.thin_q4_store(cache(), K, ks, V, vs, dtype, T, at, None, None)

    assert L.thin_q4_store(None, FAKE, None, FAKE, None, 1, 1, FAKE, None, None) == EINVAL
    assert store(K=None) == store(V=None) == store(at=None) == store(K=ODD) == EINVAL
    assert store(T=0) == store(T=(1 << 20) + 1) == store(vs=strides(640, 320, 4)) == EINVAL
    assert store(dtype=3) == EDTYPE

    def load(T=5, at=FAKE, K=FAKE, V=FAKE, dtype=1):
        return L.thin_q4_load(cache(), T, at, K, V, dtype, None)

    assert load(T=0) == load(T=(1 << 21) + 1) == load(at=None) == load(K=None) == EINVAL
    assert load(V=ODD) == EINVAL and load(dtype=-1) == EDTYPE


def test_select_refusals():
    L = _lib.lib()
    n = C.c_size_t(0)
    assert L.thin_q4_select_plan(2, 2, 1000, 3, C.byref(n)) == 0 and n.value == 4 * 3 * 16 * 8

    def select(Q=FAKE, qs=None, Hq=6, dtype=1, T=3, at=FAKE, n_sel=5, sinks=1, window=2,
               blocks=FAKE, ws=FAKE, wsb=n.value):
        return L.thin_q4_select(cache(), Q, qs, Hq, dtype, T, at, None, n_sel, sinks, window,
                                blocks, ws, wsb, None)

    assert select(Q=None) == select(Q=ODD) == select(at=None) == select(blocks=None) == EINVAL
    assert select(Hq=5) == select(Hq=0) == select(Hq=1) == select(T=0) == EINVAL
    assert select(n_sel=0) == select(n_sel=32769) == select(window=0) == EINVAL
    assert select(sinks=-1) == select(sinks=4) == select(sinks=1 << 62, window=1 << 62) == EINVAL
    assert select(qs=strides(1152, 192, 1)) == EINVAL and select(dtype=9) == EDTYPE
    assert select(ws=None) == select(wsb=n.value - 1) == select(ws=ODD) == EWORKSPACE
    assert L.thin_q4_select_plan(0, 2, 1000, 3, C.byref(n)) == EINVAL
    assert L.thin_q4_select_plan(2, 2, 1000, 3, None) == EINVAL


def test_attention_refusals():
    L = _lib.lib()
    n = C.c_size_t(0)
    assert L.thin_q4_attention_plan(2, 2, 6, 100000, 64, 3, 0, C.byref(n)) == 0 and n.value > 0

    def attend(Q=FAKE, qs=None, Hq=6, dtype=1, T=3, at=FAKE, blocks=None, n_sel=0, O=FAKE, os=None,
               ws=FAKE, wsb=n.value):
        return L.thin_q4_attention(cache(n_max=100000), Q, qs, Hq, dtype, T, at, None, blocks,
                                   n_sel, O, os, ws, wsb, None)

    assert attend(Q=None) == attend(O=None) == attend(at=None) == attend(O=ODD) == EINVAL
    assert attend(Hq=7) == attend(Hq=0) == attend(T=0) == attend(T=(1 << 20) + 1) == EINVAL
    assert attend(n_sel=3) == attend(blocks=FAKE) == attend(blocks=FAKE, n_sel=-1) == EINVAL
    assert attend(blocks=FAKE, n_sel=32769) == attend(os=strides(0, 192, 64)) == EINVAL
    assert attend(qs=strides(1, 192, 64)) == EINVAL and attend(dtype=2) == EDTYPE
    assert attend(ws=None) == attend(wsb=n.value - 1) == attend(ws=ODD) == EWORKSPACE
    for bad in [(0, 1, 1, 10, 64, 1, 0), (1, 1, 1, 10, 64, 0, 0), (1, 2, 3, 10, 64, 1, 0),
                (1, 1, 1, 10, 48, 1, 0), (1, 1, 1, 10, 64, 1, -1), (1, 1, 1025, 10, 64, 1, 0)]:
        assert L.thin_q4_attention_plan(*bad, C.byref(n)) == EINVAL
    assert L.thin_q4_attention_plan(1, 1, 1, 10, 64, 1, 0, None) == EINVAL
    # a call that does not share keys needs no workspace
    assert L.thin_q4_attention_plan(1, 1, 1, 100, 64, 1, 0, C.byref(n)) == 0 and n.value == 0


def test_turns_refusals():
    t, a = (C.c_double * 64)(), C.c_double(0)

    def turns(rot=64, base=1e4, scaling=0, factor=2.0, length=4096.0, slow=1.0, fast=32.0):
        return _lib.lib().thin_rotary_turns(rot, base, scaling, factor, length, slow, fast, t,
                                            C.byref(a))

    assert turns() == turns(scaling=1) == turns(scaling=2) == turns(scaling=3) == 0
    assert turns(factor=0.0) == 0  # ignored without scaling
    assert turns(rot=0) == turns(rot=7) == turns(base=1.0) == turns(base=math.inf) == EINVAL
    assert turns(scaling=4) == turns(scaling=-1) == turns(scaling=1, factor=0.5) == EINVAL
    assert turns(scaling=1, factor=math.nan) == turns(scaling=2, rot=2) == EINVAL
    assert turns(scaling=3, length=0.0) == turns(scaling=3, slow=32.0) == EINVAL
    assert turns(scaling=3, fast=math.nan) == EINVAL


def test_turns_follow_their_rules():
    rot, f = 64, 8.0
    plain, amp = thin_rotary_turns(rot)
    i = torch.arange(rot // 2, dtype=torch.float64)
    want = 10000.0 ** (-2 * i / rot) / (2 * math.pi)
    assert amp == 1.0 and torch.allclose(plain, want, rtol=1e-14, atol=0)
    assert torch.allclose(thin_rotary_turns(rot, scaling="linear", factor=f)[0], want / f,
                          rtol=1e-14, atol=0)
    base = thin_rotary_turns(rot, scaling="base", factor=f)[0]
    assert float(base[0]) == float(plain[0])  # the fastest pair stays
    assert math.isclose(float(base[-1]), float(plain[-1]) / f, rel_tol=1e-13)
    bands, amp = thin_rotary_turns(rot, scaling="bands", factor=f, length=4096.0)
    assert math.isclose(amp, 0.1 * math.log(f) + 1)
    n = 4096.0 * want
    assert torch.equal(bands[n >= 32], plain[n >= 32])
    assert torch.allclose(bands[n <= 1], want[n <= 1] / f, rtol=1e-14, atol=0)
    ramp = (n > 1) & (n < 32)
    assert ramp.any() and (bands[ramp] < plain[ramp]).all() and (bands[ramp] > want[ramp] / f).all()
    with pytest.raises(_lib.ThinError):
        thin_rotary_turns(rot, scaling="other")


def test_cache_buffers_are_checked():
    c = Q4Cache(2, 3, 100, 64, device="cpu")
    assert c.bounds.shape == (2, 3, 2, 2, 64) and c.k_scales.shape == (2, 3, 100, 2)
    bufs = dict(k_codes=c.k_codes, k_scales=c.k_scales, v_codes=c.v_codes, v_scales=c.v_scales,
                bounds=c.bounds)
    assert Q4Cache.over(**bufs).n_max == 100
    for name, t in [("k_codes", c.k_codes[..., :24]), ("k_scales", c.k_scales[:, :, :99]),
                    ("v_codes", c.v_codes.view(torch.int8)), ("bounds", c.bounds.float()),
                    ("v_scales", c.v_scales.transpose(0, 1)), ("k_codes", c.k_codes[0])]:
        with pytest.raises(_lib.ThinError):
            Q4Cache.over(**{**bufs, name: t})


def test_reference_encoding():
    """The reference's nearest codes: every magnitude, every tie, the scale's border."""
    x = torch.zeros(3, 32)
    x[0, :8] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0])
    x[1, :2] = torch.tensor([7.0000005, 1.0])
    codes, scales = ref.encode(x)
    assert codes[0, :8].tolist() == [0, 2, 2, 4, 4, 6, 6, 7] and scales[:, 0].tolist() == [127, 128, 2]
    assert codes[1, :2].tolist() == [6, 1]
    # nearest: no other code's value is nearer
    g = torch.Generator().manual_seed(0)
    x = torch.randn(50, 64, generator=g)
    codes, scales = ref.encode(x)
    got = ref.values(codes, scales)
    step = torch.exp2(scales.double() - 127).repeat_interleave(32, -1).unsqueeze(-1)
    best = (x.double().abs().unsqueeze(-1) - ref.GRID * step).abs().amin(-1)
    assert torch.equal((x.double() - got).abs(), best)
