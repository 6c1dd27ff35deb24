"""Sizes at the limits of the window, convolution and scan calls, answered on the host before any launch (no GPU needed)."""
import ctypes

import pytest

import paper_2606_09862_amd as bla  # noqa: F401
from test_sequence_abi import call, conv, ssm
from test_window_abi import INVALID, MUCH, OK, P, UNSUPPORTED, WORKSPACE, WS, addresses, lib  # noqa: F401


@pytest.mark.parametrize("L", [-1, 0, 7, 1 << 30, (1 << 31) - 1])
def test_single_tokens_ignore_the_length(lib, L):  # noqa: F811
    """The refusals and sizes of L = 1 for every value of a field that these calls do not use."""
    size = lambda p: lib.bla_window_step_workspace_size(ctypes.byref(p))  # noqa: E731
    assert size(P(L=L, window=5000)) == size(P(L=1, window=5000)) > 0
    tail = (WS, MUCH)
    assert call(lib.bla_window_step, P(L=L), 7, drop=[0], tail=tail) == INVALID
    assert call(lib.bla_window_step, P(L=L, window=5000), 7, tail=(None, 0)) == WORKSPACE
    assert call(lib.bla_window_step, P(L=L, B=0), 7, tail=tail) == OK
    assert call(lib.bla_conv_step, conv(L=L), 6, drop=[0]) == INVALID and call(lib.bla_conv_step, conv(L=L, B=0), 6) == OK
    assert call(lib.bla_ssm_step, ssm(L=L), 9, drop=[0]) == INVALID and call(lib.bla_ssm_step, ssm(L=L, B=0), 9) == OK
