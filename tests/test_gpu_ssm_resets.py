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


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("far", [1e12, 1e30])
def test_a_reset_past_any_sum(dtype, far):
    """Resets that no sum in float64 could hold beside the other tokens' exponents.  Their dt is as large, so they have no input."""
    _say(f"scan with resets of {far} {dtype}")
    z = inputs(82, 2, 4, 2, 150, 64, 32, dtype, True)
    for t in (2, 64, 140):
        z["dt"][:, :, t] = far / z["A"].abs()
        z["x"][:, :, t] = 0.0
    check(on_gpu(z))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rates_past_float32(dtype):
    """Heads whose dt A leaves float32's range, and one of A = -inf: y is the token's own term, and the state that of the last token."""
    bla = _bla()
    _say(f"scan with A of -3e38 and -inf {dtype}")
    B, H, G, L, d, N = 3, 4, 2, 150, 32, 16
    lengths = [150, 65, 0]
    z = inputs(83, B, H, G, L, d, N, dtype, True, lengths)
    z["A"] = torch.tensor([-3e38, -torch.inf, -2.0, -1e36])
    c = on_gpu(z)
    args = (c["x"], c["dt"], c["A"], c["Bm"], c["Cm"], c["D"])
    y, so = bla.ssm_forward(*args, state=c["state"], lengths=torch.tensor(lengths, dtype=torch.int32).cuda())
    (w, end), (s, size), live = folded({**c, "A": c["A"].clamp_min(-3e38)}, lengths, False)
    u, r = unit(dtype), share_of(N, d, L)
    close(so.flatten(0, 1), end, (r + (2.0 ** -16 if dtype == BF else 0.0)) * size, "state")
    close(y.flatten(0, 1), torch.where(live.repeat_interleave(H, 0)[..., None], w, 0.0), (u + r) * s + u * w.abs(), "y")
    one = [c[k][:2, :, 0].contiguous() for k in ("x", "dt", "Bm", "Cm")]
    state = c["state"][:2].clone()  # updated in place
    got = bla.ssm_step(one[0], one[1], c["A"], one[2], one[3], state, c["D"])
    first = {k: None if t is None else t[:2, :, :1] if k in ("x", "dt", "Bm", "Cm", "dy") else t[:2] if "state" in k else t for k, t in c.items()}
    (w, end), (s, size), _ = folded({**first, "A": c["A"].clamp_min(-3e38)}, None, False)
    close(state.flatten(0, 1), end, share_of(N, d, 1) * size, "state of a step")
    close(got.flatten(0, 1)[:, None], w, share_of(N, d, 1) * s + u * w.abs(), "y of a step")
