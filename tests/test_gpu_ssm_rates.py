"""The scan's float32 gradients that sum over all tokens (dA, dD, and ddt through its chunk) against a float32 recurrence's own error.

da_t sums the weights M_t'u dt_u of t' >= t > u.  The chunked form takes the suffix sums of M's rows minus its columns, in which the terms of u >= t
have to cancel; a recurrence never forms them.  Both round float32 sums of N d products, so over the heads the chunked form may be off by
twice as much as the recurrence run in float32 is, and by a rounding of its result.  In float32 the kernels' products sum n = max(N, d)
terms one after the other, the recurrence's sums are trees: with terms of random signs and size s a partial sum of i terms is s sqrt(i), so n roundings of
2^-24 of them leave 2^-24 s n / sqrt 2, sqrt(n / 2) of the result s sqrt(n); log2 n levels of a tree leave sqrt(log2 n) of it.  That ratio (3.0
at n = 128, 1.8 at 32) is float32's own; products of bf16 sum 32 terms at a time."""
import math

import pytest
import torch

from ssm_plain import scan
from test_gpu_parity import _bla, _say
from test_gpu_ssm import inputs

pytestmark = pytest.mark.gpu
BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64


def errors(dtype, B, H, G, L, d, N):
    """{name: (the kernels' error, the float32 recurrence's, the size of the result)}, norms over the heads."""
    bla = _bla()
    _say(f"scan rates {B}x{H}/{G}x{L}x{d} N {N} {dtype}")
    c = {k: None if t is None else t.cuda() for k, t in inputs(101, B, H, G, L, d, N, dtype, False).items()}
    _, ddt, dA, _, _, dD, _ = bla.ssm_backward(c["x"], c["dt"], c["A"], c["Bm"], c["Cm"], c["dy"], c["D"])
    ref = []
    for t in (F64, F32):
        w = {k: None if v is None else v.to(t) for k, v in c.items()}
        zero = torch.zeros(B * H, N, d, dtype=t, device="cuda")
        r = scan(w["x"].flatten(0, 1), w["dt"].flatten(0, 1), w["A"].repeat(B), w["Bm"].flatten(0, 1), w["Cm"].flatten(0, 1), w["D"].repeat(B), zero,
                 w["dy"].flatten(0, 1), zero)
        ref.append({"dA": r["dA"].reshape(B, H).sum(0), "dD": r["dD"].reshape(B, H).sum(0), "ddt": r["ddt"].reshape(B, H, L)})
    off = lambda x, k: float((x.to(F64) - ref[0][k]).norm())  # noqa: E731
    return {k: (off(x, k), off(ref[1][k], k), float(ref[0][k].norm())) for k, x in (("dA", dA), ("dD", dD), ("ddt", ddt))}


SHAPES = [(4, 8, 1, 1600, 128, 64), (2, 8, 2, 500, 64, 32), (1, 16, 1, 900, 32, 128), (3, 6, 3, 130, 128, 128)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,H,G,L,d,N", SHAPES)
def test_gradients_through_the_decays(dtype, B, H, G, L, d, N):
    e = errors(dtype, B, H, G, L, d, N)
    n = max(N, d)
    more = math.sqrt(n / 2 / math.log2(n)) if dtype == F32 else 1.0
    for k in ("dA", "ddt"):
        own, plain, size = e[k]
        assert own <= 2 * more * plain + 2.0 ** -24 * size, (k, own / size, plain / size)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,H,G,L,d,N", [*SHAPES, (16, 1, 1, 2000, 64, 16)])
def test_gradient_of_the_skip(dtype, B, H, G, L, d, N):
    """dD sums the products of x and dy over all tokens, with signs that cancel: a rounding of each product in float32 (none in bf16, whose products are
    exact), and of the result, is all that it may be off by."""
    bla = _bla()
    c = {k: None if t is None else t.cuda() for k, t in inputs(103, B, H, G, L, d, N, dtype, False).items()}
    dD = bla.ssm_backward(c["x"], c["dt"], c["A"], c["Bm"], c["Cm"], c["dy"], c["D"])[5].to(F64)
    terms = c["x"].to(F64) * c["dy"].to(F64)
    want = terms.sum((0, 2, 3))
    e = 2.0 ** -24
    # random roundings of the products: five times their root sum of squares
    bound = e * want.abs() + (5 * e * (terms ** 2).sum((0, 2, 3)).sqrt() if dtype == F32 else 1e-12 * terms.abs().sum((0, 2, 3)))
    assert float(((dD - want).abs() / bound).max()) <= 1, ((dD - want).abs() / bound).tolist()
