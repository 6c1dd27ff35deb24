"""The scan's step on its own state, at numbers of rows that the lanes of a workgroup do not divide."""
import pytest
import torch

from test_gpu_parity import _bla, _say
from test_gpu_ssm import inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("N", [8, 24, 40, 72, 104, 120])
def test_rows_that_no_pass_divides(dtype, d, N):
    """Lanes past the last row have no row to read: in place and into another buffer, step after step, the results are the same."""
    bla = _bla()
    _say(f"scan step d {d} N {N} {dtype}")
    B, H, G = 40, 6, 2
    c = {k: t.cuda() for k, t in inputs(95, B, H, G, 4, d, N, dtype, True).items()}
    own, other = c["state"].clone(), c["state"].clone()
    for t in range(4):
        x, dt, Bm, Cm = (c[k][:, :, t].contiguous() for k in ("x", "dt", "Bm", "Cm"))
        into = torch.full_like(other, torch.nan)
        y = bla.ssm_step(x, dt, c["A"], Bm, Cm, own, c["D"])
        z = bla.ssm_step(x, dt, c["A"], Bm, Cm, other, c["D"], state_out=into)
        other = into
        assert torch.equal(y, z) and torch.equal(own, other), t
