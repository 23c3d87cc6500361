"""Limits of the prompt model's calls that the other refusals do not reach (CPU only: no compute calls)."""
import ctypes

import pytest

from tests.test_api_prompt import BF16, E4M3, E_ARG, E_WORKSPACE, F16, FAKE, _kv, lib  # noqa: F401


@pytest.mark.parametrize("heads", [(1 << 23) + 1, 1 << 30, (1 << 31) - 1])
def test_more_heads_than_attention_takes(lib, heads):  # noqa: F811
    """A cache of more heads than b x q_heads may be: two rows a head, and a token's rows, are counted in 32 bits."""
    c = ctypes.byref(_kv(heads=heads, n=1))
    n = ctypes.c_size_t()
    assert lib.apc_kv_write(c, BF16, 1, FAKE, 0, 0, FAKE, 0, 0, FAKE, None) == E_ARG
    assert lib.apc_kv_read(c, BF16, 1, FAKE, FAKE, 0, 0, FAKE, 0, 0, None) == E_ARG
    assert lib.apc_attend_workspace(c, 0, heads, 4, ctypes.byref(n)) == E_ARG
    most = ctypes.byref(_kv(heads=1 << 23, n=1))
    assert lib.apc_kv_write(most, BF16, 0, FAKE, 0, 0, FAKE, 0, 0, FAKE, None) == 0
    assert lib.apc_attend_workspace(most, 1, 1 << 23, 4, ctypes.byref(n)) == 0


@pytest.mark.parametrize("dt,ks", [(F16, 0), (E4M3, 0x100000)])
def test_attend_refuses_a_workspace_that_is_none(lib, dt, ks):  # noqa: F811
    """Tables long enough to be cut need one: NULL, misaligned and short ones are refused, none is asked for short tables."""
    c = ctypes.byref(_kv(dt=dt, ks=ks, vs=ks))

    def call(pages, ws, nb, b=3):
        return lib.apc_attend(c, F16, FAKE, 256, 64, b, 4, FAKE, pages, pages, FAKE, 0, 0.125, FAKE, 256, 64, None, ws, nb, None)

    need = ctypes.c_size_t()
    assert lib.apc_attend_workspace(c, 3, 4, 2000, ctypes.byref(need)) == 0 and need.value > 0
    assert call(2000, None, need.value) == E_ARG and call(2000, ctypes.c_void_p(0x100008), need.value) == E_ARG
    assert call(2000, FAKE, need.value - 1) == E_WORKSPACE and call(2000, FAKE, 0) == E_WORKSPACE
    assert call(2000, None, 0, b=0) == 0                      # nothing to do
    assert lib.apc_attend_workspace(c, 3, 4, 4, ctypes.byref(need)) == 0 and need.value == 0
