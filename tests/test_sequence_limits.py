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


def sizes(lib, name, p):  # noqa: F811
    return getattr(lib, name)(ctypes.byref(p))


def test_window_launches(lib):  # noqa: F811
    """A launch holds fewer than 2^32 threads: shapes on both sides of that, refused before any launch and without a workspace's size."""
    tail = (WS, MUCH)
    for B, want in (((1 << 19) - 1, OK), (1 << 19, UNSUPPORTED)):             # 2^23 workgroups of 512 threads
        p = P(B=B, H=16, H_kv=4, L=64)
        assert lib.bla_window_supported(ctypes.byref(p)) == want
        assert call(lib.bla_window_forward, p, 11, drop=[0, 9, 10], tail=tail) == (INVALID if want == OK else UNSUPPORTED)
    ring = P(window=1 << 29, sinks=1 << 29)                                   # 2^35 pieces of 16 bytes in the rings after the call
    assert lib.bla_window_supported(ctypes.byref(ring)) == OK
    assert call(lib.bla_window_forward, ring, 11, drop=[0], tail=tail) == UNSUPPORTED
    assert call(lib.bla_window_forward, ring, 11, drop=[0, 9, 10], tail=tail) == INVALID
    for B, want in (((1 << 20) - 1, INVALID), (1 << 20, UNSUPPORTED)):        # 2^24 workgroups of 256 threads
        assert call(lib.bla_window_step, P(B=B, H=16, H_kv=16), 7, drop=[0], tail=tail) == want
        p = P(B=B, H=16, H_kv=16, L=64, d=128, sinks=0)
        assert call(lib.bla_window_backward, p, 10, drop=[0], tail=tail) == want
        assert (sizes(lib, "bla_window_backward_workspace_size", p) > 0) == (want == INVALID)
    p = P(B=(1 << 20) - 1, H=16, H_kv=16, L=64, d=128, sinks=4)               # ... and as many for the sinks
    assert call(lib.bla_window_backward, p, 10, drop=[0], tail=tail) == UNSUPPORTED and sizes(lib, "bla_window_backward_workspace_size", p) == 0
    p = P(B=1 << 20, H=16, H_kv=16)
    assert sizes(lib, "bla_window_step_workspace_size", p) == 0


def test_conv_launches(lib):  # noqa: F811
    most = 1 << 30
    for p in (conv(B=most, H=2, L=most, d=1 << 24), conv(B=most, H=2, L=most, d=8), conv(B=most, H=1, L=32, d=1 << 24)):
        assert lib.bla_conv_supported(ctypes.byref(p)) == UNSUPPORTED and sizes(lib, "bla_conv_backward_workspace_size", p) == 0
    for B, want in (((1 << 20) - 1, INVALID), (1 << 20, UNSUPPORTED)):        # 2^24 workgroups of the backward pass
        p = conv(B=B, H=16, L=1, d=8)
        assert lib.bla_conv_supported(ctypes.byref(p)) == OK
        assert call(lib.bla_conv_forward, p, 7, drop=[0]) == call(lib.bla_conv_step, p, 6, drop=[0]) == INVALID
        assert call(lib.bla_conv_backward, p, 11, drop=[0], tail=(WS, MUCH)) == want
        assert (sizes(lib, "bla_conv_backward_workspace_size", p) > 0) == (want == INVALID)
    p = conv(B=1, H=1 << 12, L=1, d=1 << 14, taps=8)                          # 2^26 channels with nine sums each, eight threads to a sum
    assert lib.bla_conv_supported(ctypes.byref(p)) == OK
    assert call(lib.bla_conv_backward, p, 11, drop=[0], tail=(WS, MUCH)) == UNSUPPORTED


def test_ssm_launches(lib):  # noqa: F811
    for B, want in (((1 << 20) - 1, OK), (1 << 20, UNSUPPORTED)):
        p = ssm(B=B, H=16, G=1, L=64, d=32, N=8)
        no_x = INVALID if want == OK else UNSUPPORTED
        assert lib.bla_ssm_supported(ctypes.byref(p)) == want
        assert call(lib.bla_ssm_forward, p, 10, drop=[0], tail=(WS, MUCH)) == no_x
        assert call(lib.bla_ssm_step, p, 9, drop=[0]) == no_x
    for B, want in (((1 << 19) - 1, INVALID), (1 << 19, UNSUPPORTED)):        # two walks of 2^23 workgroups
        p = ssm(B=B, H=16, G=1, L=64, d=32, N=8)
        assert call(lib.bla_ssm_backward, p, 17, drop=[0], tail=(WS, MUCH)) == want
        assert (sizes(lib, "bla_ssm_backward_workspace_size", p) > 0) == (want == INVALID)


def test_no_query_heads(lib):  # noqa: F811
    """H = 0 beside key heads or groups: refused where the call has outputs of theirs to write."""
    tail = (WS, MUCH)
    for heads, want in ((2, UNSUPPORTED), (0, OK)):
        p, s = P(H=0, H_kv=heads), ssm(H=0, G=heads)
        assert lib.bla_window_supported(ctypes.byref(p)) == lib.bla_ssm_supported(ctypes.byref(s)) == OK
        assert call(lib.bla_window_forward, p, 11, tail=tail) == want
        assert call(lib.bla_window_forward, p, 11, drop=[9, 10], tail=tail) == OK
        assert call(lib.bla_window_step, p, 7, tail=tail) == want
        assert call(lib.bla_window_backward, p, 10, tail=tail) == want
        assert call(lib.bla_ssm_backward, s, 17, tail=tail) == want
        assert call(lib.bla_ssm_forward, s, 10, tail=tail) == call(lib.bla_ssm_step, s, 9) == OK
    for p, s in ((P(H=0, B=0), ssm(H=0, B=0)), (P(H=0, L=0), ssm(H=0, L=0))):
        assert call(lib.bla_window_backward, p, 10, tail=tail) == call(lib.bla_ssm_backward, s, 17, tail=tail) == OK
