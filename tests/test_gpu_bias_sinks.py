"""Window attention with a learned bias where whole tiles are sinks far ahead of the window: their distances are not those of their places in the walk, and
lie beyond the last edge while their places do not.  The table of near distances in LDS ends behind the last edge, so a tile that took its biases
there would read what an earlier kernel left: a call whose table is full of large biases goes first.
"""
import pytest
import torch

from test_gpu_bias import BF, F32, LOG, check_backward, check_forward
from test_gpu_parity import _bla

pytestmark = pytest.mark.gpu
FULL = tuple(range(16, 1024, 16))  # 63 edges, as far as a table goes


def leave_large_biases(B, H, Hkv, L, d, dtype, pos=None):
    bla = _bla()
    z = lambda *s: torch.zeros(*s, device="cuda", dtype=dtype)  # noqa: E731
    x, bias = (z(B, H, L, d), z(B, Hkv, L, d), z(B, Hkv, L, d)), torch.full((H, len(FULL) + 1), 300.0, device="cuda")
    if pos is not None:
        ring = z(B, Hkv, 64, d)
        bla.bias_forward(*x, bias, FULL, 60, 4, pos=torch.tensor(pos, device="cuda"), cache_k=ring, cache_v=ring)
        return
    o, lse, _, _ = bla.bias_forward(*x, bias, FULL, 60, 4, want_lse=True)
    bla.bias_backward(*x, o, lse, x[0], bias, FULL, 60, 4)


SHAPES = [
    (1, 2, 1, 1000, 64, 64, 64, (32, 128)),
    (1, 2, 1, 700, 32, 16, 32, (32, 128)),       # a half tile
    (1, 2, 2, 700, 128, 1, 33, (32, 128)),       # ... and a tile that holds the window's one key too
    (1, 2, 1, 1400, 64, 100, 70, (16, 256)),     # distances beyond the table
    (1, 2, 1, 700, 64, 64, 64, LOG + (150, 300, 301)),
    (9, 16, 16, 520, 64, 48, 64, (32, 128)),     # two tiles of queries to a wave
]


def edges_of(spec):
    return _bla().bias_edges(*spec) if len(spec) == 2 else spec


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,H,Hkv,L,d,window,sinks,spec", SHAPES)
def test_forward(dtype, B, H, Hkv, L, d, window, sinks, spec):
    leave_large_biases(B, H, Hkv, L, d, dtype)
    check_forward(B, H, Hkv, L, d, window, sinks, dtype, edges_of(spec))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("L,window,sinks", [(70, 64, 64), (1, 16, 33), (200, 1, 32)])
def test_forward_from_rings(dtype, L, window, sinks):
    pos = [40, 130, 500, 900, 1 << 40]
    for spec in ((32, 128), LOG + (150, 300, 301)):
        leave_large_biases(5, 4, 2, L, 64, dtype, pos)
        check_forward(5, 4, 2, L, 64, window, sinks, dtype, edges_of(spec), pos=pos, cached=True)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,H,Hkv,L,d,window,sinks,spec", SHAPES)
def test_backward(dtype, B, H, Hkv, L, d, window, sinks, spec):
    leave_large_biases(B, H, Hkv, L, d, dtype)
    check_backward(B, H, Hkv, L, d, window, sinks, dtype, edges_of(spec))
