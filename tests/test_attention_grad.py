"""The gradient of coreset attention without a GPU: refusals before any launch, launch shapes,
and the reference against differences."""
import ctypes as C
import math
import os
import subprocess

import pytest
import torch

import attention_grad_reference as ref
from paper_2606_10944_amd import _lib

EINVAL, EDTYPE, EWORKSPACE = _lib.THIN_EINVAL, _lib.THIN_EDTYPE, _lib.THIN_EWORKSPACE
FAKE = C.c_void_p(0x10000)  # never dereferenced: every call below fails validation
ODD, BYTE = C.c_void_p(0x10008), C.c_void_p(0x10001)


def call(**kw):
    out = [C.c_void_p(0x100000 * i) for i in range(1, 4)]
    a = dict(Q=FAKE, K=FAKE, V=FAKE, dtype=1, B=2, H=3, n_q=100, n=50, d=64, idx=FAKE, logw=None,
             n_out=20, dO=FAKE, out_dtype=0, dQ=out[0], dK=out[1], dV=out[2], dlogw=None, ws=FAKE,
             wn=1 << 40)
    a.update(kw)
    return _lib.lib().thin_attention_backward(*a.values(), None)


@pytest.mark.parametrize("kw,want", [
    (dict(Q=None), EINVAL), (dict(K=None), EINVAL), (dict(V=ODD), EINVAL), (dict(dO=ODD), EINVAL),
    (dict(dQ=None), EINVAL), (dict(dK=ODD), EINVAL), (dict(dV=None), EINVAL),
    (dict(idx=None), EINVAL), (dict(idx=BYTE), EINVAL), (dict(logw=BYTE), EINVAL),
    (dict(dlogw=BYTE), EINVAL), (dict(dQ=FAKE), EINVAL), (dict(dV=FAKE), EINVAL),
    (dict(dK=C.c_void_p(0x100000)), EINVAL), (dict(dtype=2), EDTYPE), (dict(out_dtype=-1), EDTYPE),
    (dict(d=96), EINVAL), (dict(B=0), EINVAL), (dict(B=300, H=300), EINVAL), (dict(n_q=0), EINVAL),
    (dict(n=0), EINVAL), (dict(n_out=0), EINVAL), (dict(n_q=(1 << 29) // 6 + 1), EINVAL),
    (dict(n_out=(1 << 18) + 1), EINVAL), (dict(B=16, H=16, n_out=1 << 18), EINVAL), (dict(n=(1 << 30) + 1), EINVAL),
    (dict(B=1 << 62, H=4), EINVAL), (dict(ws=None), EWORKSPACE), (dict(ws=ODD), EWORKSPACE),
    (dict(wn=100), EWORKSPACE)])
def test_refusals(kw, want):
    assert call(**kw) == want


def test_plan():
    n = C.c_size_t(0)
    plan = _lib.lib().thin_attention_backward_plan
    assert plan(1, 2, 3, 100, 50, 64, 20, C.byref(n)) == 0 and n.value > 0
    assert call(wn=n.value - 1) == EWORKSPACE
    assert plan(1, 2, 3, 100, 50, 64, 20, None) == EINVAL
    assert plan(5, 2, 3, 100, 50, 64, 20, C.byref(n)) == EDTYPE
    assert plan(1, 2, 3, 100, 50, 96, 20, C.byref(n)) == EINVAL
    assert plan(1, 1, 1, 1 << 29, 1 << 30, 128, 1 << 18, C.byref(n)) == 0


PROBE = r"""
#include <cstdio>
#include "grad_plan.hpp"
using namespace thin;
int main() {
  const int64_t Ss[] = {1, 2, 5, 16, 64, 100, 257, 1000, 65535};
  const int64_t qs[] = {1, 31, 32, 33, 100, 1023, 4096, 16384, 65536, 1000003};
  const int64_t ks[] = {1, 16, 17, 32, 33, 64, 65, 128, 129, 192, 256, 257, 600, 5000, 300000};
  for (int64_t S : Ss) for (int64_t q : qs) for (int64_t k : ks) for (int b = 0; b < 2; ++b)
  for (int64_t d : {32, 64, 128}) for (int e = 0; e <= b; ++e) {
    const GradShape s = grad_shape(S, q, k, d, b, e);
    const int64_t steps = (q + grad_tile(b, s.waves) - 1) / grad_tile(b, s.waves);
    // every key and every step has a workgroup, none is without a step
    if (s.keys() * s.chunks < k || s.keys() * (s.chunks - 1) >= k) return 1;
    if ((int64_t)s.parts * s.run < steps || (int64_t)(s.parts - 1) * s.run >= steps) return 2;
    if (s.one != (k <= (e && d == 128 ? 192 : grad_most_keys(b))) || (s.one && s.chunks != 1)) return 3;
    if (!s.one && s.waves != 8) return 4;
    if (!b && d > 32 && s.tiles != 1) return 5;
    // threads of a launch fit 32 bits where rows and keys are within the entry point's limits
    if (S * k <= (1 << 25) && S * q <= (1 << 29) &&
        (S * s.chunks * s.parts * 64 * s.waves >= ((int64_t)1 << 32) ||
         (s.parts >= 16 && S * k * 256 >= ((int64_t)1 << 32)))) return 6;
    const int share = grad_share(S, q);
    if (share > 1 && S * ((q + 128 / share - 1) / (128 / share)) > 256) return 7;
    if (grad_zeros(s, q, 16 * q - 1, d * 4) || grad_zeros(s, 1, 100, d * 4)) return 8;
    if (s.parts < 100 && !grad_zeros(s, 1, 1 << 20, d * 2)) return 9;
  }
  puts("ok");
}
"""


def test_launch_shapes(tmp_path):
    src = tmp_path / "probe.cpp"
    src.write_text(PROBE)
    csrc = os.path.join(os.path.dirname(_lib.LIB_PATH), "csrc")
    exe = str(tmp_path / "probe")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", csrc, str(src), "-o", exe], check=True)
    assert subprocess.run([exe], capture_output=True, text=True).stdout.strip() == "ok"


def test_reference_against_autograd():
    g = torch.Generator()
    g.manual_seed(3)
    Q, K, V, dO = (torch.randn(2, 1, r, 32, generator=g) for r in (5, 9, 9, 5))
    idx = torch.tensor([[[0, 3, 3, 8, -1]], [[7, 1, 2, 9, 5]]], dtype=torch.int32)
    logw = torch.randn(2, 1, 5, generator=g)
    logw[0, 0, 0] = -math.inf
    x = [t.double().requires_grad_() for t in (Q, K, V, logw)]
    k, v, there = ref.coreset(x[1], x[2], idx, logw)
    o, _, _ = ref.forward(x[0], k, v, torch.where(there, x[3], -math.inf))
    (o * dO.double()).sum().backward()
    want = ref.gradient(Q, K, V, idx, logw, dO)
    for t, name in zip(x, ("dQ", "dK", "dV", "dlogw")):
        grad = torch.where(there, t.grad, 0.0) if name == "dlogw" else t.grad
        assert torch.allclose(grad, want[name][0], rtol=1e-12, atol=1e-13), name
