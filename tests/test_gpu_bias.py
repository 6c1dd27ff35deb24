"""Window attention with a learned bias on the GPU against its definition in float64 (past_plain)."""
import math

import pytest
import torch

from past_plain import row
from test_gpu_parity import _bla, _say
from test_gpu_window import dev, normal
from window_plain import close, ring_after, unit

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
LOG = (1, 2, 3, 4, 5, 6, 7, 8, 10, 13, 17, 23, 30, 40, 52)  # eight single distances, then wider buckets
FAR = (300, 301, 310, 400, 900, 901)                        # all edges beyond the table of near distances


def check_forward(B, H, Hkv, L, d, window, sinks, dtype, edges, seed=0, lengths=None, pos=None, cached=False, t0=0, scale=None, bias=None):
    bla = _bla()
    _say(f"bias forward {B}x{H}/{Hkv}x{L}x{d} window {window} sinks {sinks} {dtype} edges {edges[:3]}.. {len(edges)} lengths {lengths} pos {pos} cached {cached}")
    q, k, v = normal(seed, B, H, L, d, dtype=dtype, std=1.5), normal(seed + 1, B, Hkv, L, d, dtype=dtype), normal(seed + 2, B, Hkv, L, d, dtype=dtype)
    bias = normal(seed + 9, H, len(edges) + 1, dtype=F32, std=2.0) if bias is None else bias
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
    gq, gk, gv, gck, gcv, gl, gp, gb = dev(q, k, v, ck, cv, tl, tp, bias)
    o, lse, ok, ov = bla.bias_forward(gq, gk, gv, gb, edges, window, sinks, t0=t0, scale=scale, lengths=gl, pos=gp, cache_k=gck, cache_v=gcv,
                                      want_lse=True, want_cache=True)
    torch.cuda.synchronize()
    o, lse, ok, ov = o.cpu(), lse.cpu(), ok.cpu(), ov.cpu()
    sc = 1 / math.sqrt(d) if scale is None else scale
    u = unit(dtype)
    for b in range(B):
        p = t0 if pos is None else pos[b]
        n = 0 if p < 0 else L if lengths is None else min(max(lengths[b], 0), L)
        assert not o[b, :, n:].any() and torch.equal(lse[b, :, n:], torch.full_like(lse[b, :, n:], -math.inf))
        old = [None if x is None else x[b] for x in (ck, cv)]
        if n:
            ref = row(q[b, :, :n], k[b, :, :n], v[b, :, :n], p, window, sinks, sc, *old, bias=bias, edges=edges)
            close(o[b, :, :n], ref["o"], (u + ref["r"]) * ref["spread"] + u * ref["o"].abs(), f"o[{b}]")
            none = torch.isinf(ref["lse"])
            assert torch.equal(torch.isinf(lse[b, :, :n]), none)
            z = lambda x: torch.where(none, 0.0, x)  # noqa: E731
            close(z(lse[b, :, :n]), z(ref["lse"]), ref["r"] + 2.0 ** -22 * (1 + z(ref["lse"]).abs()), f"lse[{b}]")
        blank = torch.zeros(Hkv, sinks + window, d, dtype=dtype)
        for got, before, new in ((ok[b], old[0], k[b]), (ov[b], old[1], v[b])):
            want = ring_after(blank if before is None else before, new[:, :n], max(p, 0), window, sinks)
            assert torch.equal(got.nan_to_num(7.0), want.nan_to_num(7.0))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,H,Hkv,L,d,window,sinks,edges", [
    (1, 1, 1, 1, 32, 1, 0, (1,)),             # one token that sees itself
    (2, 4, 2, 65, 64, 65, 0, ()),             # one bucket: attention
    (2, 4, 1, 200, 64, 60, 3, LOG),           # sinks beyond every edge and before it
    (1, 6, 2, 130, 128, 64, 4, (0, 0, 5, 5)),  # buckets without a distance
    (2, 3, 3, 257, 32, 300, 1, LOG),
    (1, 2, 1, 1300, 64, 2000, 7, FAR),        # edges past the table
    (1, 4, 4, 333, 128, 100, 70, LOG + (99, 150, 220, 300)),
    (1, 2, 2, 190, 64, 17, 190, LOG),         # every key is a sink
    (9, 16, 16, 520, 64, 520, 4, tuple(range(1, 64))),  # 64 buckets, enough blocks for 128 queries to a workgroup
])
def test_forward(dtype, B, H, Hkv, L, d, window, sinks, edges):
    check_forward(B, H, Hkv, L, d, window, sinks, dtype, edges)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("L,window,sinks,pos", [
    (1, 40, 4, [0, 3, 44, 45, 1000]),
    (70, 40, 4, [0, 2, 44, 90, 1 << 40]),
    (129, 200, 0, [0, 199, 200, 201, 5000]),
    (64, 1000, 5, [4, 6, 1004, 1500, -1]),
])
def test_forward_from_rings(dtype, L, window, sinks, pos):
    check_forward(5, 4, 2, L, 64, window, sinks, dtype, LOG, pos=pos, cached=True)
    check_forward(5, 4, 2, L, 64, window, sinks, dtype, (150, 3000, 1 << 29), pos=pos, cached=True)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_forward_padded_rows_and_parts(dtype):
    check_forward(6, 4, 2, 150, 64, 50, 4, dtype, LOG, lengths=[150, 0, 1, 64, 149, -3])
    check_forward(3, 2, 1, 90, 32, 30, 2, dtype, LOG, lengths=[90, 7, 500], pos=[12, 0, 77], cached=True)
    check_forward(2, 2, 1, 5, 64, 4000, 4, dtype, LOG + FAR, pos=[3990, 9000], cached=True)  # few queries: parts of the keys
    check_forward(2, 2, 2, 100, 32, 20, 10, dtype, LOG, t0=5)
    check_forward(2, 2, 1, 150, 64, 40, 4, dtype, LOG, scale=-0.3)


def hidden(H, n, seed=3):
    """Biases of which some hide their distances, by minus infinity or the type's lowest value."""
    bias = normal(seed, H, n, dtype=F32)
    bias[0] = -math.inf                       # no key at all
    if H > 1:
        bias[1, : n // 2] = torch.finfo(F32).min
    if H > 2:
        bias[2, n // 2:] = -math.inf
    return bias


@pytest.mark.parametrize("hide", [-1.1e6, -1e10, -1e20, -3e38, -math.inf])
def test_mask_values(hide):
    """Far distances hidden by what programs use for it: the keys that come first in a row's walk have no weight, nothing overflows."""
    bias = normal(4, 2, 16, dtype=F32)
    bias[:, 12:] = hide
    bias[1, 3] = hide
    check_forward(1, 2, 1, 400, 64, 400, 0, BF, LOG, bias=bias)
    check_forward(1, 2, 1, 2, 64, 3000, 0, BF, LOG, pos=[2500], cached=True, bias=bias)
    check_backward(1, 2, 1, 200, 64, 200, 0, BF, LOG, bias=bias)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_hidden_distances(dtype):
    check_forward(2, 3, 3, 200, 64, 150, 3, dtype, LOG, bias=hidden(3, 16))
    check_forward(2, 4, 4, 3, 64, 3000, 3, dtype, LOG, pos=[2990, 9000], cached=True, bias=hidden(4, 16))


def check_backward(B, H, Hkv, L, d, window, sinks, dtype, edges, seed=50, lengths=None, scale=None, bias=None):
    bla = _bla()
    _say(f"bias backward {B}x{H}/{Hkv}x{L}x{d} window {window} sinks {sinks} {dtype} edges {edges[:3]}.. {len(edges)} lengths {lengths}")
    q, k, v = normal(seed, B, H, L, d, dtype=dtype, std=1.5), normal(seed + 1, B, Hkv, L, d, dtype=dtype), normal(seed + 2, B, Hkv, L, d, dtype=dtype)
    dO = normal(seed + 3, B, H, L, d, dtype=dtype)
    bias = normal(seed + 9, H, len(edges) + 1, dtype=F32, std=2.0) if bias is None else bias
    if lengths is not None:
        for b in range(B):
            for x in (q, k, v, dO):
                x[b, :, max(0, lengths[b]):] = math.nan
    tl = None if lengths is None else torch.tensor(lengths, dtype=torch.int32)
    gq, gk, gv, gd, gl, gb = dev(q, k, v, dO, tl, bias)
    o, lse, _, _ = bla.bias_forward(gq, gk, gv, gb, edges, window, sinks, scale=scale, lengths=gl, want_lse=True)
    args = (gq, gk, gv, o, lse, gd, gb, edges, window, sinks)
    got = bla.bias_backward(*args, scale=scale, lengths=gl)
    again = bla.bias_backward(*args, scale=scale, lengths=gl)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, again))  # a fixed order of sums
    dq, dk, dv, db = (x.cpu() for x in got)
    sc = 1 / math.sqrt(d) if scale is None else scale
    u = unit(dtype)
    want, bound = torch.zeros(H, len(edges) + 1, dtype=torch.float64), torch.zeros(H, len(edges) + 1, dtype=torch.float64)
    for b in range(B):
        n = L if lengths is None else min(max(lengths[b], 0), L)
        assert not dq[b, :, n:].any() and not dk[b, :, n:].any() and not dv[b, :, n:].any()
        if not n:
            continue
        ref = row(q[b, :, :n], k[b, :, :n], v[b, :, :n], 0, window, sinks, sc, bias=bias, edges=edges, dO=dO[b, :, :n])
        sq, sk = ref["slack"](u)
        close(dq[b, :, :n], ref["dq"], sq + u * ref["dq"].abs(), f"dq[{b}]")
        close(dk[b, :, :n], ref["dk"], sk + u * ref["dk"].abs(), f"dk[{b}]")
        close(dv[b, :, :n], ref["dv"], (u + ref["r"]) * ref["dv_spread"] + u * ref["dv"].abs(), f"dv[{b}]")
        want += ref["db"]
        bound += ref["db_bound"]
    close(db, want, bound + 2.0 ** -24 * want.abs(), "dbias")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,H,Hkv,L,d,window,sinks,edges", [
    (1, 1, 1, 1, 32, 1, 0, (1,)),
    (2, 4, 2, 65, 64, 1, 0, ()),
    (1, 6, 2, 130, 128, 64, 4, (0, 0, 5, 5)),
    (2, 3, 3, 257, 32, 300, 1, LOG),
    (1, 2, 1, 300, 64, 500, 7, LOG + FAR),
    (1, 2, 1, 1300, 64, 2000, 0, FAR),
    (1, 4, 4, 333, 128, 100, 70, LOG + (99, 150, 220, 300)),
    (1, 2, 2, 190, 64, 17, 190, LOG),
    (1, 4, 1, 1100, 64, 40, 130, LOG + (60, 61, 500, 900)),  # sinks in two key blocks, their queries in parts, several of their buckets
    (3, 4, 2, 400, 32, 400, 0, tuple(range(1, 64))),
])
def test_backward(dtype, B, H, Hkv, L, d, window, sinks, edges):
    check_backward(B, H, Hkv, L, d, window, sinks, dtype, edges)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_backward_padded_rows_and_hidden_distances(dtype):
    check_backward(6, 4, 2, 150, 64, 50, 4, dtype, LOG, lengths=[150, 0, 1, 64, 149, -3])
    check_backward(2, 2, 1, 600, 128, 50, 4, dtype, LOG, lengths=[333, 600], scale=-0.11)
    check_backward(2, 4, 2, 200, 64, 60, 3, dtype, LOG, bias=hidden(4, 16))


def test_backward_against_differences():
    """Central differences of sum(o w) in the bias, one bucket at a time: errors of 2^-24 n / h and h^2 of the sum's terms, both far below 2e-3 of the gradient's size."""
    bla = _bla()
    B, H, Hkv, L, d, window, sinks = 1, 4, 2, 70, 32, 20, 3
    x = [normal(9 + i, B, h, L, d, dtype=F32).cuda() for i, h in enumerate((H, Hkv, Hkv))]
    w, bias = normal(20, B, H, L, d, dtype=F32).cuda(), normal(21, H, 16, dtype=F32).cuda()
    o, lse, _, _ = bla.bias_forward(*x, bias, LOG, window, sinks, want_lse=True)
    db = bla.bias_backward(*x, o, lse, w, bias, LOG, window, sinks)[3].double()
    h, size = 2.0 ** -7, float((db ** 2).sum().sqrt())
    for u in range(16):
        f = []
        for s in (h, -h):
            y = bias.clone()
            y[:, u] += s
            f.append((bla.bias_forward(*x, y, LOG, window, sinks)[0].double() * w.double()).sum((0, 2, 3)))
        num = (f[0] - f[1]) / (2 * h)
        assert float((num - db[:, u]).abs().max()) < 2e-3 * size, u


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("H,Hkv,d,window,sinks,pos,edges", [
    (4, 4, 64, 40, 4, [0, 1, 3, 4, 43, 44, 45, 5000], LOG),
    (8, 1, 32, 1, 0, [0, 1, 2, 77], (0, 1)),
    (40, 2, 128, 129, 3, [0, 131, 132, 133, 1 << 50], LOG + FAR),  # twenty heads to a key head: two groups
    (4, 2, 64, 3000, 70, [2999, 3069, 3070, 100000], LOG + FAR),   # parts of the ring, blocks of sinks alone
    (2, 2, 128, 300, 0, [-1, 5, 299, -(1 << 62)], LOG),            # rows without a token
    (4, 2, 64, 954, 6, [959, 40, 960, 90000], LOG + FAR),          # the longest ring of one launch, and the next
    (4, 2, 64, 955, 6, [959, 40, 961, 90000], LOG + FAR),
    (4, 2, 64, 474, 6, [479, 40, 480, 90000], LOG + FAR),          # in float32
    (4, 2, 64, 2040, 8, [2047, 40, 2048, 90000] * 17, LOG + FAR),  # with more rows
    (4, 2, 64, 2041, 8, [2047, 40, 2049, 90000] * 17, LOG + FAR),
    (3, 3, 64, 100, 40, [20, 39, 40, 200], tuple(range(1, 64))),
])
def test_step(dtype, H, Hkv, d, window, sinks, pos, edges):
    bla = _bla()
    B = len(pos)
    _say(f"bias step {B}x{H}/{Hkv}x{d} window {window} sinks {sinks} pos {pos} {dtype}")
    q, k, v = normal(3, B, H, d, dtype=dtype, std=1.5), normal(4, B, Hkv, d, dtype=dtype), normal(5, B, Hkv, d, dtype=dtype)
    ck, cv = normal(6, B, Hkv, sinks + window, d, dtype=dtype), normal(7, B, Hkv, sinks + window, d, dtype=dtype)
    bias = normal(8, H, len(edges) + 1, dtype=F32, std=2.0)
    bias[-1, 0] = -math.inf
    for b in range(B):
        n = min(max(pos[b], 0), sinks + window)
        ck[b, :, n:], cv[b, :, n:] = math.nan, math.nan
    gq, gk, gv, gck, gcv, gp, gb = dev(q, k, v, ck, cv, torch.tensor(pos, dtype=torch.int64), bias)
    o = bla.bias_step(gq, gk, gv, gb, edges, window, sinks, gck, gcv, pos=gp)
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
        ref = row(q[b, :, None], k[b, :, None], v[b, :, None], pos[b], window, sinks, 1 / math.sqrt(d), ck[b], cv[b], bias=bias, edges=edges)
        close(o[b].cpu()[:, None], ref["o"], (u + ref["r"]) * ref["spread"] + u * ref["o"].abs(), f"o[{b}]")
