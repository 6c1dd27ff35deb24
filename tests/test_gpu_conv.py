"""The short causal convolution on the GPU against its definition in float64.

Bounds.  The kernels compute in float32 and round once to the io type (u = finfo.eps / 2).  A pre-activation z is a sum of K products and is
off by at most e = (K + 2) 2^-24 (sum |w x| + |b|); SiLU has a slope of at most 1.1 and costs some units of its own, and of the
exponent's argument:  |y - y*| <= 1.1 e + (8 + |z|) 2^-24 |y| + u |y|.  Its second derivative is at most 1/2, so
dz = dy silu'(z) is off by at most e' = |dy| (e / 2 + (16 + |z|)(1 + |z|) 2^-24), and the sums over dz by the sums over e' and n 2^-24 of
their terms' sizes.
"""
import math

import pytest
import torch

from test_gpu_parity import _bla, _say
from window_plain import close, unit

pytestmark = pytest.mark.gpu
BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64
E = 2.0 ** -24


def normal(seed, *shape, dtype=F32, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(dtype)


def plain(x, w, bias, state, silu, dy=None, dso=None):
    """One row of real tokens x [H,n,d], state [H,K-1,d]: exact results and bounds."""
    H, n, d = x.shape
    K = w.shape[2]
    x, w = x.to(F64), w.to(F64)
    bias = torch.zeros(H, d, dtype=F64) if bias is None else bias.to(F64)
    line = torch.cat([torch.zeros(H, K - 1, d, dtype=F64) if state is None else state.to(F64), x], 1)
    z = bias[:, None] + sum(line[:, j:j + n] * w[:, None, :, j] for j in range(K))
    size = bias[:, None].abs() + sum((line[:, j:j + n] * w[:, None, :, j]).abs() for j in range(K))
    ez = (K + 2) * E * size
    s = torch.sigmoid(z)
    y = z * s if silu else z
    got = {"y": y, "ey": 1.1 * ez + (8 + z.abs()) * E * y.abs(), "state": line[:, n:]}
    if dy is not None:
        dy = dy.to(F64)
        dz = dy * (s * (1 + z * (1 - s)) if silu else 1.0)
        e = dy.abs() * (0.5 * ez + (16 + z.abs()) * (1 + z.abs()) * E) if silu else torch.zeros_like(dz)
        dl, el = torch.zeros_like(line), torch.zeros_like(line)
        dw, ew = torch.zeros_like(w), torch.zeros_like(w)
        for j in range(K):
            dl[:, j:j + n] += dz * w[:, None, :, j]
            el[:, j:j + n] += (e + (K + 2) * E * dz.abs()) * w[:, None, :, j].abs()
            dw[:, :, j] = (dz * line[:, j:j + n]).sum(1)
            ew[:, :, j] = ((e + (n + 8) * E * dz.abs()) * line[:, j:j + n].abs()).sum(1)
        if dso is not None:
            dl[:, n:] += dso.to(F64)
        got.update(dx=dl[:, K - 1:], ex=el[:, K - 1:] + E * dl[:, K - 1:].abs(), dsi=dl[:, :K - 1], esi=el[:, :K - 1] + 2 * E * dl[:, :K - 1].abs(),
                   dw=dw, ew=ew, db=dz.sum(1), eb=(e + (n + 8) * E * dz.abs()).sum(1))
    return got


CASES = [
    # B, H, L, d, taps, silu, bias, state, lengths
    (1, 1, 1, 8, 1, True, True, False, None),
    (2, 3, 70, 64, 4, True, True, True, None),
    (2, 1, 33, 40, 3, False, True, True, None),              # channel threads that do not fill their power of two
    (1, 2, 300, 520, 2, True, False, False, None),           # several blocks of channels
    (4, 2, 130, 32, 4, True, True, True, [130, 0, 1, 2]),    # rows shorter than the taps
    (3, 2, 90, 128, 8, True, True, True, [90, 5, -4]),
    (2, 2, 600, 64, 7, False, True, False, [555, 600]),
    (1, 2, 0, 64, 4, True, True, True, None),                # no token: the state goes through
    (64, 8, 513, 64, 4, True, True, True, None),             # the long segments
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,H,L,d,K,silu,has_bias,has_state,lengths", CASES)
def test_forward_and_backward(dtype, B, H, L, d, K, silu, has_bias, has_state, lengths):
    bla = _bla()
    _say(f"conv {B}x{H}x{L}x{d} taps {K} silu {silu} {dtype} lengths {lengths}")
    x, dy = normal(1, B, H, L, d, dtype=dtype), normal(2, B, H, L, d, dtype=dtype)
    w = normal(3, H, d, K, std=1 / math.sqrt(K))
    bias = normal(4, H, d, std=0.5) if has_bias else None
    state, dso = (normal(5, B, H, K - 1, d), normal(6, B, H, K - 1, d)) if has_state else (None, None)
    if lengths is not None:
        for b in range(B):
            x[b, :, max(0, lengths[b]):], dy[b, :, max(0, lengths[b]):] = math.nan, math.nan
    c = lambda t: None if t is None else t.cuda()  # noqa: E731
    gl = None if lengths is None else torch.tensor(lengths, dtype=torch.int32).cuda()
    gx, gw, gb, gs, gd, gds = c(x), c(w), c(bias), c(state), c(dy), c(dso)
    y, so = bla.conv_forward(gx, gw, gb, silu=silu, state=gs, lengths=gl)
    got = bla.conv_backward(gx, gw, gd, gb, silu=silu, state=gs, dstate=gds, lengths=gl)
    again = bla.conv_backward(gx, gw, gd, gb, silu=silu, state=gs, dstate=gds, lengths=gl)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, again))
    y, so = y.cpu(), so.cpu()
    dx, dw, db, dsi = (t.cpu() for t in got)
    u = unit(dtype)
    rows = range(B) if B <= 8 else (0, 17, B - 1)
    tw = [torch.zeros(H, d, K, dtype=F64), torch.zeros(H, d, K, dtype=F64), torch.zeros(H, d, dtype=F64), torch.zeros(H, d, dtype=F64)]
    for b in range(B):
        n = L if lengths is None else min(max(lengths[b], 0), L)
        ref = plain(x[b, :, :n], w, bias, None if state is None else state[b], silu, dy[b, :, :n], None if dso is None else dso[b])
        for t, name in zip(tw, ("dw", "ew", "db", "eb")):
            t += ref[name]
        if b not in rows:
            continue
        assert not y[b, :, n:].any() and not dx[b, :, n:].any()
        assert torch.equal(so[b].to(F64), ref["state"])
        if n:
            close(y[b, :, :n], ref["y"], ref["ey"] + u * ref["y"].abs(), f"y[{b}]")
            close(dx[b, :, :n], ref["dx"], ref["ex"] + u * ref["dx"].abs(), f"dx[{b}]")
        if K > 1:
            close(dsi[b], ref["dsi"], ref["esi"], f"dstate[{b}]")
    more = (B * L + 64) * E  # the sums over rows and parts
    if L:
        close(dw, tw[0], tw[1] * (1 + more) + more * tw[0].abs() + tw[1] / max(L, 1) * B, "dw")
        close(db, tw[2], tw[3] * (1 + more) + more * tw[2].abs() + tw[3] / max(L, 1) * B, "db")
    else:
        assert not dw.any() and not db.any()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,H,d,K,silu", [(1, 1, 8, 1, True), (5, 3, 64, 4, True), (2, 2, 40, 8, False), (3, 1, 520, 2, True)])
def test_step(dtype, B, H, d, K, silu):
    bla = _bla()
    x, w, bias, state = normal(1, B, H, d, dtype=dtype), normal(2, H, d, K), normal(3, H, d), normal(4, B, H, K - 1, d)
    kept, into = state.cuda(), torch.empty_like(state).cuda()
    y0 = bla.conv_step(x.cuda(), w.cuda(), kept, bias.cuda(), silu=silu, state_out=into)
    assert torch.equal(kept.cpu(), state)
    y = bla.conv_step(x.cuda(), w.cuda(), kept, bias.cuda(), silu=silu)   # in place
    assert torch.equal(y, y0) and torch.equal(kept, into)
    u = unit(dtype)
    for b in range(B):
        ref = plain(x[b][:, None], w, bias, state[b], silu)
        close(y[b].cpu()[:, None], ref["y"], ref["ey"] + u * ref["y"].abs(), f"y[{b}]")
        assert torch.equal(into[b].cpu().to(F64), ref["state"])


def test_prompt_then_tokens():
    """Pieces of a sequence and single tokens give the outputs of one call, bit for bit in float32."""
    bla = _bla()
    B, H, L, d, K = 2, 3, 40, 64, 4
    x, w, bias = normal(1, B, H, L, d).cuda(), normal(2, H, d, K).cuda(), normal(3, H, d).cuda()
    whole, end = bla.conv_forward(x, w, bias)
    got, state, at = [], None, 0
    for n in (2, 1, 20):
        y, state = bla.conv_forward(x[:, :, at:at + n].contiguous(), w, bias, state=state)
        got.append(y)
        at += n
    while at < L:
        got.append(bla.conv_step(x[:, :, at].contiguous(), w, state, bias)[:, :, None])
        at += 1
    assert torch.equal(torch.cat(got, 2), whole) and torch.equal(state, end)
