"""Window attention with sinks on the GPU against its definition in float64 (window_plain)."""
import math

import pytest
import torch

from test_gpu_parity import _bla, _say
from window_plain import close, forward_row, ring_after, unit

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def normal(seed, *shape, dtype=BF, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(dtype)


def dev(*xs):
    return [None if x is None else x.cuda() for x in xs]


def check_forward(B, H, Hkv, L, d, window, sinks, dtype, seed=0, lengths=None, pos=None, cached=False, t0=0, scale=None):
    bla = _bla()
    _say(f"window forward {B}x{H}/{Hkv}x{L}x{d} window {window} sinks {sinks} {dtype} lengths {lengths} pos {pos} cached {cached}")
    q, k, v = normal(seed, B, H, L, d, dtype=dtype, std=1.5), normal(seed + 1, B, Hkv, L, d, dtype=dtype), normal(seed + 2, B, Hkv, L, d, dtype=dtype)
    ck = cv = None
    if cached:  # slots that no token has reached hold NaN: they are not read
        ck, cv = normal(seed + 3, B, Hkv, sinks + window, d, dtype=dtype), normal(seed + 4, B, Hkv, sinks + window, d, dtype=dtype)
        for b in range(B):
            n = min(max((pos or [t0] * B)[b], 0), sinks + window)
            ck[b, :, n:], cv[b, :, n:] = math.nan, math.nan
    if lengths is not None:  # padding is not read
        for b in range(B):
            for x in (q, k, v):
                x[b, :, max(0, lengths[b]):] = math.nan
    tl = None if lengths is None else torch.tensor(lengths, dtype=torch.int32)
    tp = None if pos is None else torch.tensor(pos, dtype=torch.int64)
    gq, gk, gv, gck, gcv, gl, gp = dev(q, k, v, ck, cv, tl, tp)
    keep = [x.clone() for x in (gq, gk, gv)]
    o, lse, ok, ov = bla.window_forward(gq, gk, gv, window, sinks, t0=t0, scale=scale, lengths=gl, pos=gp, cache_k=gck, cache_v=gcv,
                                        want_lse=True, want_cache=True)
    torch.cuda.synchronize()
    for x, y in zip((gq, gk, gv), keep):
        assert torch.equal(x.nan_to_num(7.0), y.nan_to_num(7.0))
    o, lse, ok, ov = o.cpu(), lse.cpu(), ok.cpu(), ov.cpu()
    sc = 1 / math.sqrt(d) if scale is None else scale
    u = unit(dtype)
    for b in range(B):
        p = t0 if pos is None else pos[b]
        n = 0 if p < 0 else L if lengths is None else min(max(lengths[b], 0), L)
        assert not o[b, :, n:].any() and torch.equal(lse[b, :, n:], torch.full_like(lse[b, :, n:], -math.inf))
        old = [None if x is None else x[b] for x in (ck, cv)]
        if n:
            ref = forward_row(q[b, :, :n], k[b, :, :n], v[b, :, :n], p, window, sinks, sc, *old)
            close(o[b, :, :n], ref["o"], (u + ref["r"]) * ref["spread"] + u * ref["o"].abs(), f"o[{b}]")
            close(lse[b, :, :n], ref["lse"], ref["r"] + 2.0 ** -22 * (1 + ref["lse"].abs()), f"lse[{b}]")
        blank = torch.zeros(Hkv, sinks + window, d, dtype=dtype)
        for got, before, new in ((ok[b], old[0], k[b]), (ov[b], old[1], v[b])):
            want = ring_after(blank if before is None else before, new[:, :n], max(p, 0), window, sinks)
            assert torch.equal(got.nan_to_num(7.0), want.nan_to_num(7.0))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,H,Hkv,L,d,window,sinks", [
    (1, 1, 1, 1, 32, 1, 0),            # one token that sees itself
    (2, 4, 2, 65, 64, 1, 0),           # a window of one: o = v
    (2, 4, 1, 200, 64, 1, 3),          # ... and sinks
    (1, 6, 2, 130, 128, 64, 4),        # window as long as a tile
    (2, 3, 3, 257, 32, 63, 1),         # odd sizes
    (1, 2, 1, 300, 64, 500, 7),        # a window longer than the sequence: causal attention
    (1, 4, 4, 333, 128, 100, 70),      # sinks over more than a tile
    (1, 2, 2, 190, 64, 17, 190),       # every key is a sink
    (9, 16, 16, 520, 64, 33, 4),       # enough blocks for 128 queries to a workgroup
])
def test_forward(dtype, B, H, Hkv, L, d, window, sinks):
    check_forward(B, H, Hkv, L, d, window, sinks, dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("L,window,sinks,pos", [
    (1, 40, 4, [0, 3, 44, 45, 1000]),
    (70, 40, 4, [0, 2, 44, 90, 1 << 40]),      # the call overwrites the whole ring
    (129, 200, 0, [0, 199, 200, 201, 5000]),
    (33, 1, 0, [0, 1, 2, 3, 4]),
    (64, 1000, 5, [4, 6, 1004, 1500, -1]),     # a row without tokens
])
def test_forward_from_rings(dtype, L, window, sinks, pos):
    check_forward(5, 4, 2, L, 64, window, sinks, dtype, pos=pos, cached=True)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_forward_padded_rows(dtype):
    check_forward(6, 4, 2, 150, 64, 50, 4, dtype, lengths=[150, 0, 1, 64, 149, -3])
    check_forward(3, 2, 1, 90, 32, 30, 2, dtype, lengths=[90, 7, 500], pos=[12, 0, 77], cached=True)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_forward_parts(dtype):
    """Few queries over a long ring: the keys of a block in parts."""
    check_forward(2, 2, 1, 5, 64, 4000, 4, dtype, pos=[3990, 9000], cached=True)
    check_forward(1, 1, 1, 700, 32, 2500, 0, dtype, lengths=[650])
    check_forward(2, 3, 1, 3, 128, 3001, 9, dtype, pos=[0, -5], cached=True)


def test_forward_positions_without_rings():
    """Tokens from a later position on with nothing before them: those below `sinks` are sinks."""
    check_forward(2, 2, 2, 100, 32, 20, 10, F32, t0=5)
    check_forward(2, 2, 2, 100, 32, 20, 10, BF, t0=300)


@pytest.mark.parametrize("scale", [-0.3, 2.0, 1e-6])
def test_forward_scales(scale):
    check_forward(2, 2, 1, 150, 64, 40, 4, BF, scale=scale)
    check_forward(1, 2, 1, 150, 64, 40, 4, F32, scale=scale)


def check_backward(B, H, Hkv, L, d, window, sinks, dtype, seed=50, lengths=None, scale=None):
    bla = _bla()
    _say(f"window backward {B}x{H}/{Hkv}x{L}x{d} window {window} sinks {sinks} {dtype} lengths {lengths}")
    q, k, v = normal(seed, B, H, L, d, dtype=dtype, std=1.5), normal(seed + 1, B, Hkv, L, d, dtype=dtype), normal(seed + 2, B, Hkv, L, d, dtype=dtype)
    dO = normal(seed + 3, B, H, L, d, dtype=dtype)
    if lengths is not None:
        for b in range(B):
            for x in (q, k, v, dO):
                x[b, :, max(0, lengths[b]):] = math.nan
    tl = None if lengths is None else torch.tensor(lengths, dtype=torch.int32)
    gq, gk, gv, gd, gl = dev(q, k, v, dO, tl)
    o, lse, _, _ = bla.window_forward(gq, gk, gv, window, sinks, scale=scale, lengths=gl, want_lse=True)
    dq, dk, dv = bla.window_backward(gq, gk, gv, o, lse, gd, window, sinks, scale=scale, lengths=gl)
    again = bla.window_backward(gq, gk, gv, o, lse, gd, window, sinks, scale=scale, lengths=gl)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip((dq, dk, dv), again))  # a fixed order of sums
    dq, dk, dv = dq.cpu(), dk.cpu(), dv.cpu()
    sc = 1 / math.sqrt(d) if scale is None else scale
    u = unit(dtype)
    for b in range(B):
        n = L if lengths is None else min(max(lengths[b], 0), L)
        assert not dq[b, :, n:].any() and not dk[b, :, n:].any() and not dv[b, :, n:].any()
        if not n:
            continue
        ref = forward_row(q[b, :, :n], k[b, :, :n], v[b, :, :n], 0, window, sinks, sc, dO=dO[b, :, :n])
        sq, sk = ref["slack"](u)
        close(dq[b, :, :n], ref["dq"], sq + u * ref["dq"].abs(), f"dq[{b}]")
        close(dk[b, :, :n], ref["dk"], sk + u * ref["dk"].abs(), f"dk[{b}]")
        close(dv[b, :, :n], ref["dv"], (u + ref["r"]) * ref["dv_spread"] + u * ref["dv"].abs(), f"dv[{b}]")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,H,Hkv,L,d,window,sinks", [
    (1, 1, 1, 1, 32, 1, 0),
    (2, 4, 2, 65, 64, 1, 0),
    (1, 6, 2, 130, 128, 64, 4),
    (2, 3, 3, 257, 32, 63, 1),
    (1, 2, 1, 300, 64, 500, 7),
    (1, 4, 4, 333, 128, 100, 70),
    (1, 2, 2, 190, 64, 17, 190),
    (1, 4, 1, 1100, 64, 40, 130),      # sinks in two key blocks, their queries in parts
])
def test_backward(dtype, B, H, Hkv, L, d, window, sinks):
    check_backward(B, H, Hkv, L, d, window, sinks, dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_backward_padded_rows(dtype):
    check_backward(6, 4, 2, 150, 64, 50, 4, dtype, lengths=[150, 0, 1, 64, 149, -3])
    check_backward(2, 2, 1, 600, 128, 50, 4, dtype, lengths=[333, 600], scale=-0.11)


def test_backward_against_differences():
    """Directional derivatives of sum(o w) by central differences of the float32 forward: an error of 2^-24 n / h of
    the sum's terms and h^2 of the third derivative, both far below 2e-3 of the gradient's own size here."""
    bla = _bla()
    B, H, Hkv, L, d, window, sinks = 1, 4, 2, 70, 32, 20, 3
    x = [normal(9 + i, B, h, L, d, dtype=F32).cuda() for i, h in enumerate((H, Hkv, Hkv))]
    w = normal(20, B, H, L, d, dtype=F32).cuda()
    o, lse, _, _ = bla.window_forward(*x, window, sinks, want_lse=True)
    grads = bla.window_backward(*x, o, lse, w, window, sinks)
    for i in range(3):
        step = normal(30 + i, *x[i].shape, dtype=F32).cuda()
        h = 2.0 ** -8
        f = []
        for s in (h, -h):
            y = list(x)
            y[i] = x[i] + s * step
            f.append(float((bla.window_forward(*y, window, sinks)[0].double() * w.double()).sum()))
        num, ana = (f[0] - f[1]) / (2 * h), float((grads[i].double() * step.double()).sum())
        size = float((grads[i].double() ** 2).sum().sqrt())
        assert abs(num - ana) < 2e-3 * size, (i, num, ana, size)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("H,Hkv,d,window,sinks,pos", [
    (4, 4, 64, 40, 4, [0, 1, 3, 4, 43, 44, 45, 5000]),
    (8, 1, 32, 1, 0, [0, 1, 2, 77]),
    (40, 2, 128, 129, 3, [0, 131, 132, 133, 1 << 50]),      # twenty heads to a key head: two groups
    (4, 2, 64, 3000, 4, [2999, 3003, 3004, 100000]),        # parts of the ring
    (2, 2, 128, 300, 0, [-1, 5, 299, -(1 << 62)]),          # rows without a token
])
def test_step(dtype, H, Hkv, d, window, sinks, pos):
    bla = _bla()
    B = len(pos)
    _say(f"window step {B}x{H}/{Hkv}x{d} window {window} sinks {sinks} pos {pos} {dtype}")
    q, k, v = normal(3, B, H, d, dtype=dtype, std=1.5), normal(4, B, Hkv, d, dtype=dtype), normal(5, B, Hkv, d, dtype=dtype)
    ck, cv = normal(6, B, Hkv, sinks + window, d, dtype=dtype), normal(7, B, Hkv, sinks + window, d, dtype=dtype)
    for b in range(B):
        n = min(max(pos[b], 0), sinks + window)
        ck[b, :, n:], cv[b, :, n:] = math.nan, math.nan
    gq, gk, gv, gck, gcv, gp = dev(q, k, v, ck, cv, torch.tensor(pos, dtype=torch.int64))
    o = bla.window_step(gq, gk, gv, window, sinks, gck, gcv, pos=gp)
    torch.cuda.synchronize()
    u = unit(dtype)
    for b in range(B):
        n = 0 if pos[b] < 0 else 1
        for got, before, new in ((gck[b].cpu(), ck[b], k[b]), (gcv[b].cpu(), cv[b], v[b])):
            want = ring_after(before, new[:, None][:, :n], max(pos[b], 0), window, sinks)
            assert torch.equal(got.nan_to_num(7.0), want.nan_to_num(7.0))
        if not n:
            assert not o[b].any()
            continue
        ref = forward_row(q[b, :, None], k[b, :, None], v[b, :, None], pos[b], window, sinks, 1 / math.sqrt(d), ck[b], cv[b])
        close(o[b].cpu()[:, None], ref["o"], (u + ref["r"]) * ref["spread"] + u * ref["o"].abs(), f"o[{b}]")


def test_prompt_then_tokens():
    """A prompt in uneven pieces and single tokens after it: the outputs of one call over everything."""
    bla = _bla()
    B, H, Hkv, L, d, window, sinks = 2, 4, 2, 120, 64, 30, 3
    q, k, v = (normal(70 + i, B, h, L, d, dtype=F32).cuda() for i, h in enumerate((H, Hkv, Hkv)))
    whole = bla.window_forward(q, k, v, window, sinks)[0].cpu().double()
    ck = cv = None
    got, at = [], 0
    for n in (1, 40, 2, 50):
        part = [x[:, :, at:at + n].contiguous() for x in (q, k, v)]
        o, _, ck, cv = bla.window_forward(*part, window, sinks, t0=at, cache_k=ck, cache_v=cv, want_cache=True)
        got.append(o)
        at += n
    pos = torch.full((B,), at, dtype=torch.int64, device="cuda")
    while at < L:
        got.append(bla.window_step(*(x[:, :, at].contiguous() for x in (q, k, v)), window, sinks, ck, cv, pos=pos)[:, :, None])
        pos += 1
        at += 1
    got = torch.cat(got, 2).cpu().double()
    ref = [forward_row(q[b].cpu(), k[b].cpu(), v[b].cpu(), 0, window, sinks, 1 / math.sqrt(d)) for b in range(B)]
    bound = torch.stack([(2.0 ** -24 + r["r"]) * r["spread"] + 2.0 ** -24 * r["o"].abs() for r in ref])
    close(got, torch.stack([r["o"] for r in ref]), bound, "pieces")
    close(whole, torch.stack([r["o"] for r in ref]), bound, "whole")
