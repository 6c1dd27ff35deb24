"""Window attention's bf16 gradients where few keys share a row: the roundings that they may hold, as norms.

The kernels round dS to bf16 before its products with k and q, and dq and dk at the end; the oracle counts both on these inputs (dS rounded in
float64, and the results).  They are independent, so together the error is the root of the sum of their squares.  A quarter more allows for P's
own roundings in float32 and for chance; a delta formed from outputs in bf16 and left like that adds a third to four fifths."""
import math

import pytest
import torch

from test_gpu_parity import _bla, _say
from test_gpu_window import dev, normal

pytestmark = pytest.mark.gpu
BF, F64 = torch.bfloat16, torch.float64


def counted(q, k, dO, v, n, window, sinks):
    """(dq, dk, their errors' squares) of one row's n tokens."""
    H, Hkv, d = q.shape[0], k.shape[0], q.shape[-1]
    q, k, v, dO = (t[:, :n].to(F64) for t in (q, k, v, dO))
    kh, vh = k.repeat_interleave(H // Hkv, 0), v.repeat_interleave(H // Hkv, 0)
    gap = torch.arange(n)[:, None] - torch.arange(n)[None]
    seen = (gap >= 0) & ((gap < window) | (torch.arange(n)[None] < sinks))
    P = torch.softmax((q @ kh.transpose(1, 2) / math.sqrt(d)).masked_fill(~seen, -math.inf), -1)
    dP = dO @ vh.transpose(1, 2)
    dS = P * (dP - (P * dP).sum(-1, keepdim=True)) / math.sqrt(d)
    rounded = dS.to(BF).to(F64)
    share = lambda t: t.reshape(Hkv, H // Hkv, n, d).sum(1)  # noqa: E731
    out = []
    for f in (lambda s: s @ kh, lambda s: share(s.transpose(1, 2) @ q)):
        want = f(dS)
        out.append((want, float(((f(rounded) - want) ** 2).sum()) + float(((want.to(BF).to(F64) - want) ** 2).sum())))
    return out


@pytest.mark.parametrize("B,H,Hkv,L,d,window,sinks,lengths", [
    (6, 8, 2, 16, 64, 500, 4, None),
    (10, 16, 8, 17, 32, 40, 0, None),
    (2, 12, 2, 600, 64, 8, 0, [600, 411]),
    (6, 8, 8, 24, 128, 100, 64, [24, 20, 1, 24, 13, 9]),
    (1, 4, 1, 500, 128, 8, 2, None),
    (3, 2, 1, 333, 32, 12, 1, None),
    (2, 4, 4, 64, 64, 300, 0, None),
    (4, 6, 3, 130, 64, 10, 6, [130, 0, 64, 129]),
])
def test_few_keys(B, H, Hkv, L, d, window, sinks, lengths):
    bla = _bla()
    _say(f"window backward {B}x{H}/{Hkv}x{L}x{d} window {window} sinks {sinks} lengths {lengths}")
    q, k, v, dO = (normal(110 + i, B, h, L, d, std=1.5 if i == 0 else 1.0) for i, h in enumerate((H, Hkv, Hkv, H)))
    tl = None if lengths is None else torch.tensor(lengths, dtype=torch.int32)
    gq, gk, gv, gd, gl = dev(q, k, v, dO, tl)
    o, lse, _, _ = bla.window_forward(gq, gk, gv, window, sinks, lengths=gl, want_lse=True)
    got = [t.cpu().to(F64) for t in bla.window_backward(gq, gk, gv, o, lse, gd, window, sinks, lengths=gl)[:2]]
    off, may = [0.0, 0.0], [0.0, 0.0]
    for b in range(B):
        n = L if lengths is None else lengths[b]
        if n:
            for i, (want, e) in enumerate(counted(q[b], k[b], dO[b], v[b], n, window, sinks)):
                off[i] += float(((got[i][b, :, :n] - want) ** 2).sum())
                may[i] += e
    for i, name in enumerate(("dq", "dk")):
        ratio = math.sqrt(off[i] / may[i])
        assert ratio <= 1.25, (name, ratio)
