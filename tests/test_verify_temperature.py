"""kvr_verify_drafts refuses, on the host, a temperature that it cannot divide
by; 0 is not taken for 1."""
import ctypes

import pytest

from paper_2608_15797_gb300 import kvr

lib = kvr.lib
ONE = ctypes.c_void_p(16)


def status(temperature):
    d = kvr.kvr_verify_desc(2, 3, 100, temperature, kvr.KVR_BF16)
    need = lib.kvr_verify_workspace_bytes(ctypes.byref(d))
    # a workspace that is too small: nothing is launched in either case
    got = lib.kvr_verify_drafts(ctypes.byref(d), ONE, 100, ONE, 100, ONE, ONE,
                                ONE, None, ONE, ONE, ONE, 0, None)
    return need, got


@pytest.mark.parametrize("temperature", [0.0, -0.0, -1.0, 1e-45, 4e-39,
                                         float("inf"), float("nan")])
def test_refused(temperature):
    assert status(temperature) == (0, kvr.KVR_EINVAL)


@pytest.mark.parametrize("temperature", [1e-38, 1e-5, 0.7, 1.0, 3e38])
def test_taken(temperature):
    need, got = status(temperature)
    assert need > 0 and got == kvr.KVR_ENOMEM
