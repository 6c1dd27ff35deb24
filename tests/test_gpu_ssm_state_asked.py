"""The selective scan's outputs, whether the state after the call is asked for or not, in one segment and in several."""
import pytest
import torch

from ssm_plain import share_of
from test_gpu_parity import _bla, _say
from test_gpu_ssm import inputs
from test_gpu_ssm_paths import folded, on_gpu
from window_plain import close, unit

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,H,G,L,d,N", [
    (2, 2, 1, 200, 64, 128),                 # one segment
    (1, 2, 1, 64 * 40 + 5, 32, 24),          # nine
    (2, 16, 2, 64 * 16 + 9, 64, 64),         # four
    (3, 4, 1, 64 * 12, 128, 128),
])
def test_outputs_do_not_depend_on_it(dtype, B, H, G, L, d, N):
    """A weight that enters the state with fewer bits than float32's would show: a term from an earlier chunk is rounded once, with the state where y
    reads it, as a term of the own chunk is with its weight."""
    bla = _bla()
    _say(f"scan {B}x{H}/{G}x{L}x{d} N {N} {dtype}")
    z = inputs(91, B, H, G, L, d, N, dtype, True)
    z["A"] = -torch.rand(H, generator=torch.Generator().manual_seed(92)) * 100.0 / L
    c = on_gpu(z)
    args = (c["x"], c["dt"], c["A"], c["Bm"], c["Cm"], c["D"])
    y, so = bla.ssm_forward(*args, state=c["state"])
    y0, none = bla.ssm_forward(*args, state=c["state"], want_state=False)
    assert none is None and torch.equal(y, y0)
    (w, end), (s, size), _ = folded(c, None, False)
    u, r = unit(dtype), share_of(N, d, L)
    close(y.flatten(0, 1), w, (u + r) * s + u * w.abs(), "y")
    close(so.flatten(0, 1), end, (r + (2.0 ** -16 if dtype == torch.bfloat16 else 0.0)) * size, "state")
