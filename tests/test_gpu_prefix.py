"""Window attention behind a shared prefix on the GPU against its definition in float64 (past_plain)."""
import math

import pytest
import torch

from past_plain import row
from test_gpu_parity import _bla, _say
from test_gpu_window import dev, normal
from window_plain import close, ring_after, unit

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def prefixes(G, Hkv, P, d, dtype, plen, seed):
    """Prefixes whose tokens past their lengths hold NaN: they are not read."""
    pk, pv = normal(seed, G, Hkv, P, d, dtype=dtype), normal(seed + 1, G, Hkv, P, d, dtype=dtype)
    n = [P if plen is None else min(max(plen[g], 0), P) for g in range(G)]
    for g in range(G):
        pk[g, :, n[g]:], pv[g, :, n[g]:] = math.nan, math.nan
    return pk, pv, n


def check_forward(B, G, H, Hkv, L, d, P, window, sinks, dtype, plen=None, lengths=None, pos=None, cached=False, seed=0, scale=None):
    bla = _bla()
    _say(f"prefix forward {B}/{G}x{H}/{Hkv}x{L}x{d} P {P} window {window} sinks {sinks} {dtype} plen {plen} lengths {lengths} pos {pos} cached {cached}")
    q, k, v = normal(seed, B, H, L, d, dtype=dtype, std=1.5), normal(seed + 1, B, Hkv, L, d, dtype=dtype), normal(seed + 2, B, Hkv, L, d, dtype=dtype)
    pk, pv, np = prefixes(G, Hkv, P, d, dtype, plen, seed + 5)
    ck = cv = None
    if cached:
        ck, cv = normal(seed + 3, B, Hkv, sinks + window, d, dtype=dtype), normal(seed + 4, B, Hkv, sinks + window, d, dtype=dtype)
        for b in range(B):
            n = min(max((pos or [0] * B)[b], 0), sinks + window)
            ck[b, :, n:], cv[b, :, n:] = math.nan, math.nan
    if lengths is not None:
        for b in range(B):
            for x in (q, k, v):
                x[b, :, max(0, lengths[b]):] = math.nan
    t = lambda x, ty: None if x is None else torch.tensor(x, dtype=ty)  # noqa: E731
    gq, gk, gv, gck, gcv, gpk, gpv, gl, gp, gn = dev(q, k, v, ck, cv, pk, pv, t(lengths, torch.int32), t(pos, torch.int64), t(plen, torch.int32))
    o, lse, ok, ov = bla.prefix_forward(gq, gk, gv, gpk, gpv, window, sinks, scale=scale, lengths=gl, pos=gp, prefix_lengths=gn, cache_k=gck,
                                        cache_v=gcv, want_lse=True, want_cache=True)
    torch.cuda.synchronize()
    o, lse, ok, ov = o.cpu(), lse.cpu(), ok.cpu(), ov.cpu()
    sc = 1 / math.sqrt(d) if scale is None else scale
    u = unit(dtype)
    for b in range(B):
        p, g = 0 if pos is None else pos[b], b // (B // G)
        n = 0 if p < 0 else L if lengths is None else min(max(lengths[b], 0), L)
        assert not o[b, :, n:].any() and torch.equal(lse[b, :, n:], torch.full_like(lse[b, :, n:], -math.inf))
        old = [None if x is None else x[b] for x in (ck, cv)]
        if n:
            ref = row(q[b, :, :n], k[b, :, :n], v[b, :, :n], p, window, sinks, sc, *old, front_k=pk[g, :, :np[g]], front_v=pv[g, :, :np[g]])
            close(o[b, :, :n], ref["o"], (u + ref["r"]) * ref["spread"] + u * ref["o"].abs(), f"o[{b}]")
            close(lse[b, :, :n], ref["lse"], ref["r"] + 2.0 ** -22 * (1 + ref["lse"].abs()), f"lse[{b}]")
        blank = torch.zeros(Hkv, sinks + window, d, dtype=dtype)
        for got, before, new in ((ok[b], old[0], k[b]), (ov[b], old[1], v[b])):
            want = ring_after(blank if before is None else before, new[:, :n], max(p, 0), window, sinks)
            assert torch.equal(got.nan_to_num(7.0), want.nan_to_num(7.0))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,G,H,Hkv,L,d,P,window,sinks,plen", [
    (1, 1, 1, 1, 1, 32, 1, 1, 0, None),
    (2, 1, 4, 2, 65, 64, 0, 40, 3, None),            # no prefix: window attention
    (4, 2, 4, 2, 65, 64, 64, 40, 3, [64, 0]),        # a prefix of one tile, another without a token
    (3, 3, 6, 2, 130, 128, 97, 64, 4, [1, 97, 33]),
    (2, 1, 2, 1, 300, 64, 1000, 500, 0, [777]),      # fewer tokens than the tensor holds
    (9, 3, 16, 16, 520, 64, 70, 33, 4, [70, -2, 500]),  # enough blocks for 128 queries to a workgroup; lengths out of range
])
def test_forward(dtype, B, G, H, Hkv, L, d, P, window, sinks, plen):
    check_forward(B, G, H, Hkv, L, d, P, window, sinks, dtype, plen)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_forward_rings_padding_parts(dtype):
    check_forward(5, 1, 4, 2, 70, 64, 130, 40, 4, dtype, pos=[0, 2, 44, 90, -1], cached=True)
    check_forward(6, 2, 4, 2, 150, 64, 31, 50, 4, dtype, plen=[31, 7], lengths=[150, 0, 1, 64, 149, -3])
    check_forward(2, 1, 2, 1, 5, 64, 4000, 300, 4, dtype, pos=[290, 9000], cached=True)  # few queries: parts of the keys
    check_forward(2, 2, 2, 1, 1, 128, 5000, 30, 0, dtype, plen=[5000, 10], scale=-0.2)
    check_forward(1, 1, 40, 2, 3, 32, 90, 30, 2, dtype)


def check_step(B, G, H, Hkv, d, P, window, sinks, pos, dtype, plen=None, seed=3, scale=None):
    bla = _bla()
    _say(f"prefix step {B}/{G}x{H}/{Hkv}x{d} P {P} window {window} sinks {sinks} pos {pos} plen {plen} {dtype}")
    pos = [pos[b % len(pos)] for b in range(B)]
    q, k, v = normal(seed, B, H, d, dtype=dtype, std=1.5), normal(seed + 1, B, Hkv, d, dtype=dtype), normal(seed + 2, B, Hkv, d, dtype=dtype)
    ck, cv = normal(seed + 3, B, Hkv, sinks + window, d, dtype=dtype), normal(seed + 4, B, Hkv, sinks + window, d, dtype=dtype)
    pk, pv, np = prefixes(G, Hkv, P, d, dtype, plen, seed + 5)
    for b in range(B):
        n = min(max(pos[b], 0), sinks + window)
        ck[b, :, n:], cv[b, :, n:] = math.nan, math.nan
    tn = None if plen is None else torch.tensor(plen, dtype=torch.int32)
    gq, gk, gv, gck, gcv, gpk, gpv, gp, gn = dev(q, k, v, ck, cv, pk, pv, torch.tensor(pos, dtype=torch.int64), tn)
    o = bla.prefix_step(gq, gk, gv, gpk, gpv, window, sinks, gck, gcv, pos=gp, prefix_lengths=gn, scale=scale)
    torch.cuda.synchronize()
    u, sc = unit(dtype), 1 / math.sqrt(d) if scale is None else scale
    for b in range(B):
        n, g = 0 if pos[b] < 0 else 1, b // (B // G)
        for got, before, new in ((gck[b].cpu(), ck[b], k[b]), (gcv[b].cpu(), cv[b], v[b])):
            want = ring_after(before, new[:, None][:, :n], max(pos[b], 0), window, sinks)
            assert torch.equal(got.nan_to_num(7.0), want.nan_to_num(7.0))
        if not n:
            assert not o[b].any()
            continue
        ref = row(q[b, :, None], k[b, :, None], v[b, :, None], pos[b], window, sinks, sc, ck[b], cv[b], front_k=pk[g, :, :np[g]], front_v=pv[g, :, :np[g]])
        close(o[b].cpu()[:, None], ref["o"], (u + ref["r"]) * ref["spread"] + u * ref["o"].abs(), f"o[{b}]")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,G,H,Hkv,d,P,window,sinks,pos,plen", [
    (1, 1, 1, 1, 32, 1, 1, 0, [0], None),
    (8, 1, 4, 4, 64, 0, 40, 4, [0, 1, 3, 4, 43, 44, 45, 5000], None),
    (4, 2, 8, 1, 32, 65, 1, 0, [0, 1, 2, 77], [65, 0]),
    (5, 1, 40, 2, 128, 300, 129, 3, [0, 131, 132, 133, 1 << 50], [299]),   # twenty heads to a key head
    (4, 1, 4, 2, 64, 3000, 2000, 4, [1999, 2003, 2004, 100000], None),     # parts of the ring and of the prefix
    (6, 3, 2, 2, 128, 130, 300, 0, [-1, 5, 299, -(1 << 62)], [130, 1, 64]),  # rows without a token
    (4, 2, 4, 2, 32, 777, 64, 4, [0, 67, 68, 500], [777, 33]),             # prefix and ring in one launch without parts, the last block of each in part
    (2, 1, 24, 1, 64, 448, 500, 12, [3, 900], None),                       # ... two groups of heads, as many blocks as it takes
    (2, 1, 2, 1, 64, 449, 500, 12, [3, 900], None),                        # ... and one more
    (4, 2, 4, 2, 64, 100, 64, 4, [0, 67, 68, -1], [0, 100]),                # ... and a prefix without tokens
    (6, 6, 4, 2, 64, 0, 3000, 0, [2999, 3, 5000], None),                   # no prefix, a long ring
    (70, 2, 8, 2, 64, 200, 33, 0, [3, 40, -1, 0, 100], [200, 63]),          # queries in several blocks, the last in part
    (40, 1, 16, 4, 64, 1111, 20, 0, [10, 25], None),
])
def test_step(dtype, B, G, H, Hkv, d, P, window, sinks, pos, plen):
    check_step(B, G, H, Hkv, d, P, window, sinks, pos, dtype, plen)


def test_step_scales():
    check_step(3, 1, 4, 2, 64, 100, 20, 2, [10, 30, 0], BF, scale=-0.3)
    check_step(3, 1, 4, 2, 64, 100, 20, 2, [10, 30, 0], F32, scale=2.0)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_prefix_then_tokens(dtype):
    """The prefix as a prompt of its own, questions behind it and single tokens: one attention over everything."""
    bla = _bla()
    B, H, Hkv, d, P, L = 3, 4, 2, 64, 100, 40
    pq, pk, pv = normal(1, 1, H, P, d, dtype=dtype), normal(2, 1, Hkv, P, d, dtype=dtype), normal(3, 1, Hkv, P, d, dtype=dtype)
    q, k, v = (normal(10 + i, B, h, L, d, dtype=dtype) for i, h in enumerate((H, Hkv, Hkv)))
    gq, gk, gv, gpk, gpv = dev(q, k, v, pk, pv)
    got, n = [], 33
    o, _, ck, cv = bla.prefix_forward(*(x[:, :, :n].contiguous() for x in (gq, gk, gv)), gpk, gpv, L, want_cache=True)
    got.append(o)
    for t in range(n, L):
        got.append(bla.prefix_step(*(x[:, :, t].contiguous() for x in (gq, gk, gv)), gpk, gpv, L, 0, ck, cv, t0=t)[:, :, None])
    got = torch.cat(got, 2).cpu()
    u = unit(dtype)
    for b in range(B):
        every = [torch.cat([x[0], y[b]], 1) for x, y in ((pq, q), (pk, k), (pv, v))]
        ref = row(*every, 0, P + L, 0, 1 / math.sqrt(d))
        close(got[b], ref["o"][:, P:], ((u + ref["r"]) * ref["spread"] + u * ref["o"].abs())[:, P:], f"row {b}")
