"""Window attention on the host (no GPU needed): shapes, workspace sizes and every refusal, before any launch."""
import ctypes

import pytest
import torch

import paper_2606_09862_amd as bla

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3


@pytest.fixture(scope="module")
def lib():
    from test_abi_cpu import os as _os
    if not _os.path.exists(bla.LIB_PATH):
        from paper_2606_09862_amd import build
        build.build()
    return bla.lib()


def P(**kw):
    base = dict(B=2, H=4, H_kv=2, L=100, d=64, window=40, sinks=4, io_dtype=1, t0=0, scale=0.0)
    base.update(kw)
    return bla.WindowParams(*base.values())


def test_struct_layout():
    # eight int32, int64, float (+ 4 bytes of tail) as in bla.h
    assert ctypes.sizeof(bla.WindowParams) == 48
    assert bla.WindowParams.t0.offset == 32 and bla.WindowParams.scale.offset == 40


@pytest.mark.parametrize("kw,expect", [
    ({}, OK), (dict(H=4, H_kv=4), OK), (dict(d=32), OK), (dict(d=128, io_dtype=0), OK), (dict(L=0), OK), (dict(B=0), OK),
    (dict(window=1, sinks=0), OK), (dict(window=1 << 29, sinks=1 << 29), OK), (dict(scale=-0.5), OK), (dict(t0=1 << 62), OK),
    (dict(d=48), UNSUPPORTED), (dict(d=256), UNSUPPORTED), (dict(window=1 << 30, sinks=1), UNSUPPORTED),
    (dict(scale=1e-7), UNSUPPORTED), (dict(scale=2e6), UNSUPPORTED), (dict(B=1 << 30, H=4, H_kv=2), UNSUPPORTED),
    (dict(H=4, H_kv=3), INVALID), (dict(H_kv=0), INVALID), (dict(H_kv=-1), INVALID), (dict(H=-4), INVALID), (dict(B=-1), INVALID),
    (dict(L=-1), INVALID), (dict(d=0), INVALID), (dict(window=0), INVALID), (dict(sinks=-1), INVALID), (dict(io_dtype=2), INVALID),
    (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(t0=-1), INVALID),
    (dict(t0=(1 << 62) + 1), INVALID),
])
def test_supported(lib, kw, expect):
    assert lib.bla_window_supported(ctypes.byref(P(**kw))) == expect
    if expect != OK:
        p = ctypes.byref(P(**kw))
        assert lib.bla_window_workspace_size(p) == 0 and lib.bla_window_backward_workspace_size(p) == 0


def test_null_params(lib):
    assert lib.bla_window_supported(None) == INVALID
    assert lib.bla_window_workspace_size(None) == lib.bla_window_step_workspace_size(None) == lib.bla_window_backward_workspace_size(None) == 0


def addresses(n):
    return [ctypes.c_void_p(0x100000000 * (i + 1)) for i in range(n)]


WS = ctypes.c_void_p(0x7000000000000)
MUCH = 1 << 40


def forward(lib, p=None, drop=(), put=(), nbytes=MUCH, ws=WS):
    # q, k, v, lengths, pos, cache_k_in, cache_v_in, o, lse, cache_k_out, cache_v_out
    a = addresses(11)
    for i in drop:
        a[i] = None
    for i, x in put:
        a[i] = ctypes.c_void_p(x)
    return lib.bla_window_forward(ctypes.byref(p or P()), *a, ws, nbytes, None)


def test_forward_refusals(lib):
    for i in (0, 1, 2, 7):                                   # q, k, v, o missing
        assert forward(lib, drop=[i]) == INVALID
    for i in (5, 6, 9, 10):                                  # one ring of two
        assert forward(lib, drop=[i]) == INVALID
    for i in (0, 1, 2, 5, 6, 7, 9, 10):                      # not 16-byte aligned
        assert forward(lib, put=[(i, 0x900000008)]) == INVALID
    assert forward(lib, put=[(3, 0x900000002)]) == INVALID   # lengths, pos, lse
    assert forward(lib, put=[(4, 0x900000004)]) == INVALID
    assert forward(lib, put=[(8, 0x900000002)]) == INVALID
    for out in (7, 9, 10):                                   # an output over an input
        for i in (0, 1, 2, 5, 6):
            assert forward(lib, put=[(i, 0x9000000000), (out, 0x9000000010)]) == INVALID
    assert forward(lib, P(H_kv=3)) == INVALID and forward(lib, P(d=48)) == UNSUPPORTED
    small = P(B=1, H=1, H_kv=1, L=4, window=5000)            # few queries, many keys: parts, so a workspace
    need = lib.bla_window_workspace_size(ctypes.byref(small))
    assert need > 0
    assert forward(lib, small, nbytes=need - 1) == WORKSPACE and forward(lib, small, ws=None) == WORKSPACE
    assert forward(lib, small, ws=ctypes.c_void_p(0x7000000000004)) == WORKSPACE
    assert forward(lib, P(B=0), drop=range(11), nbytes=0, ws=None) == OK


def test_step_refusals(lib):
    def step(p=None, drop=(), put=(), nbytes=MUCH, ws=WS):
        a = addresses(7)                                     # q, k, v, pos, cache_k, cache_v, o
        for i in drop:
            a[i] = None
        for i, x in put:
            a[i] = ctypes.c_void_p(x)
        return lib.bla_window_step(ctypes.byref(p or P()), *a, ws, nbytes, None)

    for i in (0, 1, 2, 4, 5, 6):
        assert step(drop=[i]) == INVALID
        assert step(put=[(i, 0x900000008)]) == INVALID
    assert step(put=[(3, 0x900000004)]) == INVALID
    for i in (0, 1, 2):
        for out in (4, 5, 6):
            assert step(put=[(i, 0x9000000000), (out, 0x9000000010)]) == INVALID
    assert step(put=[(4, 0x9000000000), (5, 0x9000000010)]) == INVALID
    assert step(put=[(4, 0x9000000000), (6, 0x9000000010)]) == INVALID
    p = P(window=5000)
    need = lib.bla_window_step_workspace_size(ctypes.byref(p))
    assert need > 0 and step(p, nbytes=need - 1) == WORKSPACE and step(p, ws=None) == WORKSPACE
    assert step(P(B=0), drop=range(7), ws=None, nbytes=0) == OK


def test_backward_refusals(lib):
    def back(p=None, drop=(), put=(), nbytes=MUCH, ws=WS):
        a = addresses(10)                                    # q, k, v, o, lse, dO, lengths, dq, dk, dv
        for i in drop:
            a[i] = None
        for i, x in put:
            a[i] = ctypes.c_void_p(x)
        return lib.bla_window_backward(ctypes.byref(p or P()), *a, ws, nbytes, None)

    for i in (0, 1, 2, 3, 4, 5, 7, 8, 9):
        assert back(drop=[i]) == INVALID
    for i in (0, 1, 2, 3, 5, 7, 8, 9):
        assert back(put=[(i, 0x900000008)]) == INVALID
    assert back(put=[(4, 0x900000002)]) == INVALID and back(put=[(6, 0x900000002)]) == INVALID
    for out in (7, 8, 9):
        for i in (0, 1, 2, 3, 5):
            assert back(put=[(i, 0x9000000000), (out, 0x9000000010)]) == INVALID
    assert back(put=[(8, 0x9000000000), (9, 0x9000000010)]) == INVALID
    assert back(P(t0=1)) == UNSUPPORTED
    need = lib.bla_window_backward_workspace_size(ctypes.byref(P()))
    assert need > 0 and back(nbytes=need - 1) == WORKSPACE and back(ws=None) == WORKSPACE
    assert back(P(L=0), drop=range(10), nbytes=0, ws=None) == OK


def test_binding_refusals():
    x = torch.zeros(1, 2, 8, 32)
    with pytest.raises(ValueError):                          # not on a GPU
        bla.window_forward(x, x, x, 4)
    with pytest.raises(ValueError):
        bla.window_forward(x.half(), x.half(), x.half(), 4)
