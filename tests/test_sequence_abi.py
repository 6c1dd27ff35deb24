"""The short convolution and the selective scan on the host (no GPU needed): shapes, workspace sizes and every refusal, before any
launch."""
import ctypes

import pytest
import torch

import paper_2606_09862_amd as bla
from test_window_abi import INVALID, MUCH, OK, UNSUPPORTED, WORKSPACE, WS, addresses, lib  # noqa: F401

FAR = 0x9000000000


def conv(**kw):
    base = dict(B=2, H=4, L=100, d=64, taps=4, silu=1, io_dtype=1)
    base.update(kw)
    return bla.ConvParams(*base.values())


def ssm(**kw):
    base = dict(B=2, H=4, G=2, L=100, d=64, N=64, io_dtype=1)
    base.update(kw)
    return bla.SsmParams(*base.values())


def call(fn, p, n, drop=(), put=(), tail=()):
    a = addresses(n)
    for i in drop:
        a[i] = None
    for i, x in put:
        a[i] = ctypes.c_void_p(x)
    return fn(ctypes.byref(p), *a, *tail, None)


@pytest.mark.parametrize("kw,expect", [
    ({}, OK), (dict(taps=1), OK), (dict(taps=8, silu=0, io_dtype=0), OK), (dict(d=8, H=1), OK), (dict(d=4000), OK), (dict(L=0), OK),
    (dict(B=0), OK), (dict(taps=9), UNSUPPORTED), (dict(d=12), UNSUPPORTED), (dict(d=(1 << 24) + 8), UNSUPPORTED),
    (dict(B=1 << 20, H=1 << 12), UNSUPPORTED), (dict(taps=0), INVALID), (dict(taps=-1), INVALID), (dict(silu=2), INVALID),
    (dict(io_dtype=3), INVALID), (dict(d=0), INVALID), (dict(L=-1), INVALID), (dict(B=-1), INVALID), (dict(H=-1), INVALID),
])
def test_conv_supported(lib, kw, expect):  # noqa: F811
    p = ctypes.byref(conv(**kw))
    assert lib.bla_conv_supported(p) == expect
    if expect != OK:
        assert lib.bla_conv_backward_workspace_size(p) == 0
    assert lib.bla_conv_supported(None) == INVALID


@pytest.mark.parametrize("kw,expect", [
    ({}, OK), (dict(N=8), OK), (dict(N=128, d=128, io_dtype=0), OK), (dict(d=32, N=40), OK), (dict(G=4), OK), (dict(L=0), OK), (dict(B=0), OK),
    (dict(N=136), UNSUPPORTED), (dict(N=12), UNSUPPORTED), (dict(d=48), UNSUPPORTED), (dict(L=(1 << 30) + 1), UNSUPPORTED),
    (dict(B=1 << 20, L=1 << 20), UNSUPPORTED), (dict(N=0), INVALID), (dict(G=3), INVALID), (dict(G=0), INVALID), (dict(d=0), INVALID),
    (dict(io_dtype=-1), INVALID), (dict(L=-1), INVALID), (dict(B=-1), INVALID), (dict(H=-4), INVALID),
])
def test_ssm_supported(lib, kw, expect):  # noqa: F811
    p = ctypes.byref(ssm(**kw))
    assert lib.bla_ssm_supported(p) == expect
    if expect != OK:
        assert lib.bla_ssm_workspace_size(p) == 0 and lib.bla_ssm_backward_workspace_size(p) == 0
    assert lib.bla_ssm_supported(None) == INVALID


def test_struct_layouts():
    assert ctypes.sizeof(bla.ConvParams) == 28 and ctypes.sizeof(bla.SsmParams) == 28


def test_conv_refusals(lib):  # noqa: F811
    f = lambda **k: call(lib.bla_conv_forward, k.pop("p", conv()), 7, **k)   # x, w, bias, lengths, state_in, y, state_out  # noqa: E731
    for i in (0, 1, 5):
        assert f(drop=[i]) == INVALID
    for i in (0, 1, 2, 4, 5, 6):
        assert f(put=[(i, FAR + 8)]) == INVALID
    assert f(put=[(3, FAR + 2)]) == INVALID
    for out in (5, 6):
        for i in (0, 1, 2, 4):
            assert f(put=[(i, FAR), (out, FAR + 16)]) == INVALID
    assert f(put=[(5, FAR), (6, FAR + 16)]) == INVALID
    assert f(p=conv(B=0), drop=range(7)) == OK and f(p=conv(taps=9)) == UNSUPPORTED

    s = lambda **k: call(lib.bla_conv_step, k.pop("p", conv()), 6, **k)      # x, w, bias, state_in, y, state_out  # noqa: E731
    for i in (0, 1, 3, 4, 5):
        assert s(drop=[i]) == INVALID
    for i in range(6):
        assert s(put=[(i, FAR + 8)]) == INVALID
    for out in (4, 5):
        for i in (0, 1, 2):
            assert s(put=[(i, FAR), (out, FAR + 16)]) == INVALID
    assert s(put=[(3, FAR), (5, FAR + 16)]) == INVALID                       # over the state, but not the state itself
    assert s(put=[(3, FAR), (4, FAR)]) == INVALID
    assert s(p=conv(B=0), drop=range(6)) == OK

    # x, w, bias, dy, lengths, state_in, dstate_out, dx, dw, dbias, dstate_in
    tail = (WS, MUCH)
    b = lambda **k: call(lib.bla_conv_backward, k.pop("p", conv()), 11, tail=k.pop("tail", tail), **k)  # noqa: E731
    for i in (0, 1, 3, 7, 8):
        assert b(drop=[i]) == INVALID
    for i in (0, 1, 2, 3, 5, 6, 7, 8, 9, 10):
        assert b(put=[(i, FAR + 8)]) == INVALID
    assert b(put=[(4, FAR + 2)]) == INVALID
    for out in (7, 8, 9, 10):
        for i in (0, 1, 2, 3, 5, 6):
            assert b(put=[(i, FAR), (out, FAR + 16)]) == INVALID
    assert b(put=[(7, FAR), (8, FAR + 16)]) == INVALID
    need = lib.bla_conv_backward_workspace_size(ctypes.byref(conv()))
    assert need > 0
    assert b(tail=(WS, need - 1)) == b(tail=(None, MUCH)) == b(tail=(ctypes.c_void_p(0x7000000000004), MUCH)) == WORKSPACE
    assert b(p=conv(B=0)) == UNSUPPORTED and b(p=conv(H=0), drop=range(11)) == OK


def test_ssm_refusals(lib):  # noqa: F811
    # x, dt, A, Bm, Cm, D, lengths, state_in, y, state_out
    tail = (WS, MUCH)
    f = lambda **k: call(lib.bla_ssm_forward, k.pop("p", ssm()), 10, tail=k.pop("tail", tail), **k)  # noqa: E731
    for i in (0, 1, 2, 3, 4, 8):
        assert f(drop=[i]) == INVALID
    for i in (0, 3, 4, 7, 8, 9):
        assert f(put=[(i, FAR + 8)]) == INVALID
    for i in (1, 2, 5, 6):
        assert f(put=[(i, FAR + 2)]) == INVALID
    for out in (8, 9):
        for i in (0, 1, 2, 3, 4, 5, 7):
            assert f(put=[(i, FAR), (out, FAR)]) == INVALID
    assert f(put=[(8, FAR), (9, FAR + 16)]) == INVALID
    long = ssm(L=5000)
    need = lib.bla_ssm_workspace_size(ctypes.byref(long))
    assert need > 0 and f(p=long, tail=(WS, need - 1)) == f(p=long, tail=(None, MUCH)) == WORKSPACE
    assert f(p=ssm(B=0), drop=range(10), tail=(None, 0)) == OK

    # x, dt, A, Bm, Cm, D, state_in, y, state_out
    s = lambda **k: call(lib.bla_ssm_step, k.pop("p", ssm()), 9, **k)  # noqa: E731
    for i in (0, 1, 2, 3, 4, 6, 7, 8):
        assert s(drop=[i]) == INVALID
    for i in (0, 3, 4, 6, 7, 8):
        assert s(put=[(i, FAR + 8)]) == INVALID
    for out in (7, 8):
        for i in (0, 1, 2, 3, 4, 5):
            assert s(put=[(i, FAR), (out, FAR)]) == INVALID
    assert s(put=[(6, FAR), (8, FAR + 16)]) == INVALID and s(put=[(6, FAR), (7, FAR + 16)]) == INVALID
    assert s(p=ssm(B=0), drop=range(9)) == OK

    # x, dt, A, Bm, Cm, D, dy, lengths, state_in, dstate_out, dx, ddt, dA, dB, dC, dD, dstate_in
    b = lambda **k: call(lib.bla_ssm_backward, k.pop("p", ssm()), 17, tail=k.pop("tail", tail), **k)  # noqa: E731
    for i in (0, 1, 2, 3, 4, 6, 10, 11, 12, 13, 14):
        assert b(drop=[i]) == INVALID
    for i in (0, 3, 4, 6, 8, 9, 10, 13, 14, 16):
        assert b(put=[(i, FAR + 8)]) == INVALID
    for i in (1, 2, 5, 7, 11, 12, 15):
        assert b(put=[(i, FAR + 2)]) == INVALID
    for out in (10, 11, 12, 13, 14, 15, 16):
        for i in (0, 1, 2, 3, 4, 5, 6, 8, 9):
            assert b(put=[(i, FAR), (out, FAR)]) == INVALID
    assert b(put=[(13, FAR), (14, FAR + 16)]) == INVALID
    need = lib.bla_ssm_backward_workspace_size(ctypes.byref(ssm()))
    assert need > 0 and b(tail=(WS, need - 1)) == b(tail=(None, MUCH)) == WORKSPACE
    assert b(p=ssm(B=0)) == b(p=ssm(L=0)) == UNSUPPORTED


def test_binding_refusals():
    x, w = torch.zeros(1, 2, 8, 32), torch.zeros(2, 32, 4)
    with pytest.raises(ValueError):                                          # not on a GPU
        bla.conv_forward(x, w)
    with pytest.raises(ValueError):
        bla.conv_forward(x.half(), w)
    with pytest.raises(ValueError):
        bla.conv_forward(x, torch.zeros(2, 32))
    with pytest.raises(bla.BlaError):
        bla.conv_forward(x, torch.zeros(2, 32, 9))
    dt, A, B = torch.zeros(1, 2, 8), torch.zeros(2), torch.zeros(1, 1, 8, 16)
    with pytest.raises(ValueError):
        bla.ssm_forward(x, dt, A, B, B)
    with pytest.raises(ValueError):
        bla.ssm_forward(x, dt, A, B[0], B)
    with pytest.raises(bla.BlaError):
        bla.ssm_forward(x, dt, A, torch.zeros(1, 1, 8, 12), B)
