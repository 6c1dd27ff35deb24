"""The selective scan where single tokens decay by far more than the tokens around them: the decays after such a token are differences of large sums.

Bounds as in ssm_plain: exponents between tokens that still see each other stay below 50, however large the sums are that they are differences of."""
import pytest
import torch

from ssm_plain import share_of
from test_gpu_parity import _bla, _say
from test_gpu_ssm import inputs
from test_gpu_ssm_paths import check_backward, folded, on_gpu
from window_plain import close, unit

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def check(c):
    bla = _bla()
    B, H, L, d = c["x"].shape
    N, dtype = c["Bm"].shape[-1], c["x"].dtype
    y, so = bla.ssm_forward(c["x"], c["dt"], c["A"], c["Bm"], c["Cm"], c["D"], state=c["state"])
    (w, end), (s, size), _ = folded(c, None, False)
    u, r = unit(dtype), share_of(N, d, L)
    close(so.flatten(0, 1), end, (r + (2.0 ** -16 if dtype == BF else 0.0)) * size, "state")
    close(y.flatten(0, 1), w, (u + r) * s + u * w.abs(), "y")
    check_backward(c, None)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,N", [(32, 16), (64, 128)])
@pytest.mark.parametrize("far", [1e3, 1e5, 1e6])
def test_a_reset_early_in_a_chunk(dtype, d, N, far):
    """dt A = -far at the third token of one chunk and the first of the next, with an input there and without."""
    _say(f"scan with resets of {far}, d {d} N {N} {dtype}")
    z = inputs(81, 2, 4, 2, 150, d, N, dtype, True)
    for t in (2, 64):
        z["dt"][:, :, t] = far / z["A"].abs()
        z["x"][:, ::2, t] = 0.0
    check(on_gpu(z))
