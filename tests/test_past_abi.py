"""Attention with a learned bias, behind a prefix and over a cache of bounded size on the host (no GPU needed): shapes, workspace sizes and
every refusal, before any launch; the binding against the header."""
import ctypes
import os
import re

import pytest
import torch

import paper_2606_09862_amd as bla
from test_sequence_abi import call
from test_window_abi import INVALID, MUCH, OK, P, UNSUPPORTED, WORKSPACE, WS, addresses, lib  # noqa: F401

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "bla.h")
TAIL = (WS, MUCH)


def prefix(P=100, G=1, **kw):
    base = dict(B=4, H=4, H_kv=2, L=100, d=64, window=40, sinks=4, io_dtype=1, t0=0, scale=0.0)
    base.update(kw)
    return bla.PrefixParams(bla.WindowParams(*base.values()), P, G)


def evict(**kw):
    base = dict(B=2, H=4, H_kv=2, L=100, d=64, slots=50, recent=4, io_dtype=1, t0=0, scale=0.0)
    base.update(kw)
    return bla.EvictParams(*base.values())


def edges(*x):
    return (ctypes.c_int32 * max(len(x), 1))(*x)


def test_arguments_as_in_the_header(lib):  # noqa: F811
    """Every call that the binding declares takes as many arguments as its prototype (one too few would pass a pointer as 32 bits)."""
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    seen = 0
    for name, args in re.findall(r"\b(bla_\w+)\(([^)]*)\);", text):
        fn = getattr(lib, name)
        if fn.argtypes is not None:
            assert len(fn.argtypes) == len(args.split(",")), name
            seen += 1
    assert seen > 30
    for name in ("bias_forward", "bias_step", "bias_backward", "prefix_forward", "prefix_step", "evict_forward", "evict_select", "evict_step"):
        assert getattr(lib, "bla_" + name).argtypes is not None


def test_struct_layout():
    assert ctypes.sizeof(bla.PrefixParams) == 56 and bla.PrefixParams.P.offset == 48 and bla.PrefixParams.G.offset == 52
    assert ctypes.sizeof(bla.EvictParams) == 48 and bla.EvictParams.t0.offset == 32 and bla.EvictParams.scale.offset == 40


def bias_call(lib, name, n, p=None, buckets=4, e=(1, 2, 9), drop=(), put=(), tail=TAIL):  # noqa: F811
    a = addresses(n)
    for i in drop:
        a[i] = None
    for i, x in put:
        a[i] = ctypes.c_void_p(x)
    return getattr(lib, name)(ctypes.byref(p or P()), buckets, None if e is None else edges(*e), *a, *tail, None)


CALLS = (("bla_bias_forward", 12), ("bla_bias_step", 8), ("bla_bias_backward", 12))


@pytest.mark.parametrize("name,n", CALLS)
def test_buckets(lib, name, n):  # noqa: F811
    """Refused buckets; what passes is stopped by a missing q."""
    go = lambda buckets, e: bias_call(lib, name, n, buckets=buckets, e=e, drop=[0])  # noqa: E731
    for buckets, e in ((1, None), (1, ()), (2, (0,)), (4, (0, 0, 1 << 29)), (64, tuple(range(63)))):
        assert go(buckets, e) == INVALID                      # q missing
        assert bias_call(lib, name, n, P(d=48), buckets, e) == UNSUPPORTED
    assert go(0, ()) == go(-1, ()) == go(2, None) == go(2, (-1,)) == go(3, (5, 4)) == INVALID
    assert go(65, tuple(range(64))) == go(3, (5, (1 << 29) + 1)) == UNSUPPORTED


def test_bias_refusals(lib):  # noqa: F811
    F, S, B = (lambda lib=lib, c=c, **kw: bias_call(lib, *c, **kw) for c in CALLS)
    for i in (0, 1, 2, 3, 8):                                 # q, k, v, bias, o
        assert F(drop=[i]) == INVALID
    for i in (6, 7, 10, 11):                                  # one ring of two
        assert F(drop=[i]) == INVALID
    for i in (0, 1, 2, 6, 7, 8, 10, 11):
        assert F(put=[(i, 0x900000008)]) == INVALID
    for i, x in ((3, 2), (4, 2), (5, 4), (9, 2)):             # bias, lengths, pos, lse
        assert F(put=[(i, 0x900000000 + x)]) == INVALID
    for out in (8, 9, 10, 11):
        for i in (0, 1, 2, 3, 6, 7):
            assert F(put=[(i, 0x9000000000), (out, 0x9000000010)]) == INVALID
    assert F(p=P(H_kv=3)) == INVALID and F(p=P(B=0), drop=range(12), tail=(None, 0)) == OK
    small = P(B=1, H=1, H_kv=1, L=4, window=5000)
    assert F(p=small, tail=(WS, lib.bla_window_workspace_size(ctypes.byref(small)) - 1)) == WORKSPACE and F(p=small, tail=(None, 0)) == WORKSPACE
    for i in (0, 1, 2, 3, 5, 6, 7):
        assert S(drop=[i]) == INVALID
    assert S(put=[(3, 0x900000002)]) == INVALID
    for out in (5, 6, 7):
        for i in (0, 1, 2, 3):
            assert S(put=[(i, 0x9000000000), (out, 0x9000000010)]) == INVALID
    big = P(window=5000)
    need = lib.bla_bias_step_workspace_size(ctypes.byref(big))
    assert need > 0 and S(p=big, tail=(WS, need - 1)) == WORKSPACE
    assert lib.bla_bias_step_workspace_size(ctypes.byref(P(window=956))) == 0 < lib.bla_bias_step_workspace_size(ctypes.byref(P(window=957)))  # 120 KiB of keys
    for i in (0, 1, 2, 3, 4, 5, 6, 8, 9, 10, 11):
        assert B(drop=[i]) == INVALID
    for i in (3, 5, 7, 11):                                   # bias, lse, lengths, dbias
        assert B(put=[(i, 0x900000002)]) == INVALID
    for out in (8, 9, 10, 11):
        for i in (0, 1, 2, 3, 4, 5, 6):
            assert B(put=[(i, 0x9000000000), (out, 0x9000000010)]) == INVALID
    assert B(put=[(10, 0x9000000000), (11, 0x9000000010)]) == INVALID
    assert B(p=P(t0=1)) == UNSUPPORTED
    size = lambda p, n=4: lib.bla_bias_backward_workspace_size(ctypes.byref(p), n)  # noqa: E731
    assert B(tail=(WS, size(P()) - 1)) == WORKSPACE and B(tail=(None, 0)) == WORKSPACE
    assert size(P(), 0) == size(P(), 65) == size(P(d=48)) == 0 and size(P(), 64) > size(P(), 2) > 0
    assert B(p=P(L=0), drop=range(12), tail=(None, 0)) == B(p=P(B=0), drop=range(12), tail=(None, 0)) == UNSUPPORTED  # dbias would be left unwritten
    assert B(p=P(H=0, H_kv=0), drop=range(12), tail=(None, 0)) == OK


@pytest.mark.parametrize("kw,expect", [
    ({}, OK), (dict(P=0), OK), (dict(G=4), OK), (dict(G=2, P=1), OK), (dict(B=0, G=0), OK), (dict(P=1 << 30, H_kv=1), OK),
    (dict(G=3), INVALID), (dict(G=0), INVALID), (dict(G=-1), INVALID), (dict(P=-1), INVALID), (dict(window=0), INVALID), (dict(d=48), UNSUPPORTED),
    (dict(P=(1 << 30) + 1, H_kv=1), UNSUPPORTED), (dict(P=1 << 30, G=4, H_kv=4, d=128), UNSUPPORTED), (dict(scale=1e-7), UNSUPPORTED),
])
def test_prefix_supported(lib, kw, expect):  # noqa: F811
    p = ctypes.byref(prefix(**kw))
    assert lib.bla_prefix_supported(p) == expect
    if expect != OK:
        assert lib.bla_prefix_workspace_size(p) == lib.bla_prefix_step_workspace_size(p) == 0
    assert lib.bla_prefix_supported(None) == INVALID and lib.bla_prefix_workspace_size(None) == lib.bla_prefix_step_workspace_size(None) == 0


def test_prefix_refusals(lib):  # noqa: F811
    F = lambda p=None, drop=(), put=(), tail=TAIL: call(lib.bla_prefix_forward, p or prefix(), 14, drop, put, tail)  # noqa: E731
    for i in (0, 1, 2, 3, 4, 10):                             # q, k, v, prefix_k, prefix_v, o
        assert F(drop=[i]) == INVALID and F(put=[(i, 0x900000008)]) == INVALID
    for i in (8, 9, 12, 13):
        assert F(drop=[i]) == INVALID
    assert F(put=[(5, 0x900000002)]) == INVALID               # prefix_lengths
    for out in (10, 11, 12, 13):
        for i in (0, 1, 2, 3, 4, 5, 8, 9):
            assert F(put=[(i, 0x9000000000), (out, 0x9000000000)]) == INVALID
    small = prefix(B=1, H=1, H_kv=1, L=4, P=9000)
    need = lib.bla_prefix_workspace_size(ctypes.byref(small))
    assert need > 0 and F(small, tail=(WS, need - 1)) == WORKSPACE and F(small, tail=(None, 0)) == WORKSPACE
    assert F(prefix(B=0), drop=range(14), tail=(None, 0)) == OK
    assert F(prefix(P=0), drop=[0, 3, 4]) == INVALID          # no prefix: q alone is missed
    S = lambda p=None, drop=(), put=(), tail=TAIL: call(lib.bla_prefix_step, p or prefix(), 10, drop, put, tail)  # noqa: E731
    for i in (0, 1, 2, 3, 4, 7, 8, 9):
        assert S(drop=[i]) == INVALID and S(put=[(i, 0x900000008)]) == INVALID
    assert S(put=[(5, 0x900000002)]) == S(put=[(6, 0x900000004)]) == INVALID
    for out in (7, 8, 9):
        for i in (0, 1, 2, 3, 4, 5, 6):
            assert S(put=[(i, 0x9000000000), (out, 0x9000000000)]) == INVALID
    size = lambda **kw: lib.bla_prefix_step_workspace_size(ctypes.byref(prefix(**kw)))  # noqa: E731
    need = size(P=3000)
    assert need > 0 and S(prefix(P=3000), tail=(WS, need - 1)) == S(prefix(P=3000), tail=(None, 0)) == WORKSPACE
    assert size() == size(P=0) == 0 and size(B=64) > 0        # few queries, a short prefix and ring: one launch without parts
    for L in (-1, 0, 7, (1 << 31) - 1):                       # the step ignores L
        assert size(P=3000, L=L) == need and S(prefix(L=L), drop=[0]) == INVALID


@pytest.mark.parametrize("kw,expect", [
    ({}, OK), (dict(slots=1, recent=0), OK), (dict(recent=49), OK), (dict(slots=1 << 24, L=1), OK), (dict(L=0), OK), (dict(B=0), OK),
    (dict(recent=50), INVALID), (dict(recent=-1), INVALID), (dict(slots=0, recent=0), INVALID), (dict(slots=-5), INVALID), (dict(H_kv=3), INVALID),
    (dict(L=-1), INVALID), (dict(io_dtype=2), INVALID), (dict(t0=-1), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(slots=(1 << 24) + 1), UNSUPPORTED), (dict(d=96), UNSUPPORTED), (dict(scale=3e6), UNSUPPORTED), (dict(B=1 << 20, L=1 << 10), UNSUPPORTED),
])
def test_evict_supported(lib, kw, expect):  # noqa: F811
    p = ctypes.byref(evict(**kw))
    assert lib.bla_evict_supported(p) == expect
    if expect != OK:
        assert lib.bla_evict_workspace_size(p) == 0
    assert lib.bla_evict_supported(None) == INVALID and lib.bla_evict_workspace_size(None) == lib.bla_evict_step_workspace_size(None) == 0


def test_evict_refusals(lib):  # noqa: F811
    # q, k, v, lengths, pos, cache_k, cache_v, score_in, o, lse, score_out
    F = lambda p=None, drop=(), put=(), tail=TAIL: call(lib.bla_evict_forward, p or evict(), 11, drop, put, tail)  # noqa: E731
    for i in (0, 1, 2, 5, 6, 7, 8, 10):                       # ... one of the cache's three among them
        assert F(drop=[i]) == INVALID
    for i in (0, 1, 2, 5, 6, 8):
        assert F(put=[(i, 0x900000008)]) == INVALID
    for i in (3, 7, 9, 10):
        assert F(put=[(i, 0x900000002)]) == INVALID
    for out in (8, 9, 10):
        for i in (0, 1, 2, 5, 6, 7):
            assert F(put=[(i, 0x9000000000), (out, 0x9000000010)]) == INVALID
    assert F(put=[(8, 0x9000000000), (10, 0x9000000010)]) == INVALID
    need = lib.bla_evict_workspace_size(ctypes.byref(evict()))
    assert need > 0 and F(tail=(WS, need - 1)) == F(tail=(None, 0)) == F(tail=(ctypes.c_void_p(0x7000000000004), MUCH)) == WORKSPACE
    assert F(evict(B=0), drop=range(11), tail=(None, 0)) == OK and F(evict(H=0)) == UNSUPPORTED
    # k, v, score, lengths, pos, cache_k_in, cache_v_in, at_in, cache_k_out, cache_v_out, score_out, at_out
    S = lambda p=None, drop=(), put=(): call(lib.bla_evict_select, p or evict(), 12, drop, put)  # noqa: E731
    for i in (0, 1, 2, 5, 6, 7, 8, 9, 10, 11):
        assert S(drop=[i]) == INVALID
    for i in (0, 1, 5, 6, 8, 9):
        assert S(put=[(i, 0x900000008)]) == INVALID
    for i, x in ((2, 2), (3, 2), (4, 4), (7, 4), (10, 2), (11, 4)):
        assert S(put=[(i, 0x900000000 + x)]) == INVALID
    for out in (8, 9, 10, 11):
        for i in (0, 1, 2, 5, 6, 7):
            assert S(put=[(i, 0x9000000000), (out, 0x9000000010)]) == INVALID
    assert S(put=[(8, 0x9000000000), (9, 0x9000000010)]) == INVALID
    assert S(evict(B=0), drop=range(12)) == OK and S(evict(recent=50)) == INVALID
    # q, k, v, pos, cache_k, cache_v, score_in, at_in, o, score_out, at_out
    T = lambda p=None, drop=(), put=(), tail=TAIL: call(lib.bla_evict_step, p or evict(), 11, drop, put, tail)  # noqa: E731
    for i in (0, 1, 2, 4, 5, 6, 7, 8, 9, 10):
        assert T(drop=[i]) == INVALID
    for i in (0, 1, 2, 4, 5, 8):
        assert T(put=[(i, 0x900000008)]) == INVALID
    for i, x in ((3, 4), (6, 2), (7, 4), (9, 2), (10, 4)):
        assert T(put=[(i, 0x900000000 + x)]) == INVALID
    for out in (4, 5, 8, 9, 10):
        for i in (0, 1, 2, 3):
            assert T(put=[(i, 0x9000000000), (out, 0x9000000000)]) == INVALID
    for i, out in ((6, 9), (7, 10)):                          # in place is fine (the workspace is missed), a few bytes off is not
        assert T(put=[(i, 0x9000000000), (out, 0x9000000000)], tail=(None, 0)) == WORKSPACE
        assert T(put=[(i, 0x9000000000), (out, 0x9000000010)]) == INVALID
    assert T(put=[(6, 0x9000000000), (10, 0x9000000000)]) == T(put=[(7, 0x9000000000), (9, 0x9000000000)]) == INVALID
    need = lib.bla_evict_step_workspace_size(ctypes.byref(evict()))
    assert need > 0 and T(tail=(WS, need - 1)) == WORKSPACE
    for L in (-1, 0, 7, (1 << 31) - 1):
        assert lib.bla_evict_step_workspace_size(ctypes.byref(evict(L=L))) == need and T(evict(L=L), drop=[0]) == INVALID


def test_select_takes_no_notice_of_query_heads_and_scale(lib):  # noqa: F811
    S = lambda p, drop=(): call(lib.bla_evict_select, p, 12, drop)  # noqa: E731
    for kw in (dict(H=3), dict(H=-1), dict(H=0), dict(H=1 << 30), dict(scale=float("nan")), dict(scale=3e6), dict(scale=1e-9)):
        assert S(evict(B=0, **kw), range(12)) == OK, kw
        assert S(evict(**kw), [2]) == INVALID, kw             # the missing scores, and nothing before them
    assert lib.bla_evict_select(None, *addresses(12), None) == INVALID


def test_launches(lib):  # noqa: F811
    """A launch holds fewer than 2^32 threads: refused before any launch, and without a workspace's size."""
    size = lambda name, p: getattr(lib, name)(ctypes.byref(p))  # noqa: E731
    big = P(B=1 << 20, H=16, H_kv=16, L=64, d=128, sinks=0)
    assert lib.bla_bias_backward_workspace_size(ctypes.byref(big), 4) == 0
    assert bias_call(lib, "bla_bias_backward", 12, p=big, drop=[0]) == UNSUPPORTED
    assert bias_call(lib, "bla_bias_step", 8, p=P(B=1 << 20, H=16, H_kv=16), drop=[0]) == UNSUPPORTED
    x = prefix(B=1 << 20, H=16, H_kv=16)
    assert size("bla_prefix_step_workspace_size", x) == 0 and call(lib.bla_prefix_step, x, 10, drop=[0], tail=TAIL) == UNSUPPORTED
    x = evict(B=1 << 20, H=16, H_kv=16, slots=20)
    assert size("bla_evict_step_workspace_size", x) == 0 and call(lib.bla_evict_step, x, 11, drop=[0], tail=TAIL) == UNSUPPORTED
    x = evict(B=1 << 18, H=16, H_kv=16, slots=20, L=1)
    assert call(lib.bla_evict_select, x, 12, drop=[0]) == UNSUPPORTED


def test_edges():
    """The usual buckets: half of them one distance each, the others' bounds the smallest whole numbers past a geometric progression."""
    assert bla.bias_edges(2, 1) == (1,) and bla.bias_edges(4, 16) == (1, 2, 6)   # 2 sqrt 8 = 5.66
    assert bla.bias_edges(16, 2048) == (1, 2, 3, 4, 5, 6, 7, 8, 16, 32, 64, 128, 256, 512, 1024)  # powers of two: exact
    e = bla.bias_edges(32, 128)
    assert len(e) == 31 and e[:16] == tuple(range(1, 17)) and e[-1] == 113
    for i, x in enumerate(e[16:], 1):
        assert (x / 16) ** 16 >= 8 ** i * (1 - 1e-12) and ((x - 1) / 16) ** 16 < 8 ** i
    for buckets, far in ((1, 10), (32, 15), (0, 5)):
        with pytest.raises(ValueError):
            bla.bias_edges(buckets, far)


def test_binding_refusals():
    x, y = torch.zeros(2, 2, 8, 32), torch.zeros(2, 2, 32)
    b = torch.zeros(2, 4)
    with pytest.raises(ValueError):                          # not on a GPU
        bla.bias_forward(x, x, x, b, (1, 2, 3), 4)
    with pytest.raises(ValueError):
        bla.prefix_forward(x, x, x, x, x, 4)
    with pytest.raises(ValueError):                          # not [G, H_kv, P, d]
        bla.prefix_step(y, y, y, y, y, 4, 0, x, x)
    with pytest.raises(ValueError):
        bla.evict_forward(x, x, x, 4)
    with pytest.raises(ValueError):
        bla.evict_select(x, x, torch.zeros(2, 2, 12), 4)
    with pytest.raises(ValueError):
        bla.evict_step(y, y, y, y, y, y, y)
    with pytest.raises(bla.BlaError):                        # recent >= slots
        bla.evict_select(x, x, torch.zeros(2, 2, 12), 4, recent=4)
    with pytest.raises(bla.BlaError):                        # sizes past the parameter block's fields
        bla.evict_forward(x, x, x, 1 << 33)
