"""The 4-bit cache's limits without a GPU."""
import ctypes as C

import pytest

from paper_2606_10944_amd import _lib


@pytest.mark.parametrize("B,H,T", [(1, 64, 600), (1, 8, 1 << 20), (4, 8, 32), (65535, 1, 2)])
def test_a_prompts_selection_needs_a_workspace_of_few_tokens(B, H, T):
    """Scores in LDS need none; for caches of more rows, 64 MiB (or a token's) at most,
    whatever the number of tokens."""
    plan, n = _lib.lib().thin_q4_select_plan, C.c_size_t(0)
    assert plan(B, H, 131072, T, C.byref(n)) == 0 and n.value == 0
    for rows in (131073, 1 << 20, 1 << 21):
        assert plan(B, H, rows, T, C.byref(n)) == 0
        nb = -(-rows // 64)
        assert n.value % (nb * 8) == 0 and 0 < n.value <= 64 << 20
        assert n.value == min(512, (64 << 20) // (nb * 8), B * H * T) * nb * 8


FAKE = C.c_void_p(0x10000)  # never dereferenced: every call below fails validation


@pytest.mark.parametrize("amp", [3.5e38, -1e39, 1e300])
def test_rotary_refuses_factors_that_are_no_float32(amp):
    """Rows are turned in float32: such a factor would be infinite there."""
    rc = _lib.lib().thin_rotary(FAKE, None, 4, FAKE, None, None, None, 0, None, None, 1, 2, 3, 64,
                                32, 0, FAKE, 0, FAKE, amp, 0, None)
    assert rc == _lib.THIN_EINVAL


def test_turns_refuse_a_base_that_overflows():
    """base * factor^(rot / (rot - 2)) past the float64 numbers has no table."""
    t, a = (C.c_double * 64)(), C.c_double(0)
    turns = _lib.lib().thin_rotary_turns
    assert turns(64, 1e300, 2, 1e200, 0.0, 1.0, 32.0, t, C.byref(a)) == _lib.THIN_EINVAL
    assert turns(4, 1e4, 2, 1e160, 0.0, 1.0, 32.0, t, C.byref(a)) == _lib.THIN_EINVAL
    assert turns(64, 1e4, 2, 1e200, 0.0, 1.0, 32.0, t, C.byref(a)) == 0
