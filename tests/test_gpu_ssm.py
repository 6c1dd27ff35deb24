"""The selective state space scan on the GPU against its recurrence in float64 (ssm_plain)."""
import math

import pytest
import torch

from ssm_plain import exact, share_of
from test_gpu_parity import _bla, _say
from window_plain import close, unit

pytestmark = pytest.mark.gpu
BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64


def inputs(seed, B, H, G, L, d, N, dtype, state, lengths=None, fast=False):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    z = {"x": n(B, H, L, d).to(dtype), "dy": n(B, H, L, d).to(dtype), "Bm": n(B, G, L, N).to(dtype), "Cm": n(B, G, L, N).to(dtype),
         "dt": torch.exp(torch.rand(B, H, L, generator=g) * math.log(100.0) + math.log(1e-3)),
         "A": -(torch.rand(H, generator=g) * 15 + 1), "D": torch.rand(H, generator=g) + 0.5,
         "state": 0.3 * n(B, H, N, d) if state else None, "dstate": 0.3 * n(B, H, N, d) if state else None}
    if fast:  # a decay that forgets everything within a token, and one that forgets nothing
        z["A"][0], z["A"][-1] = -5000.0, 0.0
    if lengths is not None:
        for b in range(B):
            m = max(0, lengths[b])
            for k in ("x", "dy", "Bm", "Cm", "dt"):
                z[k][b, :, m:] = math.nan
    return z


def run(z, lengths=None, D=True):
    bla = _bla()
    c = {k: None if t is None else t.cuda() for k, t in z.items()}
    gl = None if lengths is None else torch.tensor(lengths, dtype=torch.int32).cuda()
    Dm = c["D"] if D else None
    y, so = bla.ssm_forward(c["x"], c["dt"], c["A"], c["Bm"], c["Cm"], Dm, state=c["state"], lengths=gl)
    back = lambda: bla.ssm_backward(c["x"], c["dt"], c["A"], c["Bm"], c["Cm"], c["dy"], Dm, state=c["state"], dstate=c["dstate"],  # noqa: E731
                                    lengths=gl)
    got = back() if z["x"].shape[2] else None
    if got is not None:
        assert all(torch.equal(p, q) for p, q in zip(got, back()))  # a fixed order of sums
    torch.cuda.synchronize()
    return [y.cpu(), so.cpu()] + ([t.cpu() for t in got] if got is not None else [])


def check(B, H, G, L, d, N, dtype, state=False, lengths=None, seed=1, D=True, fast=False):
    _say(f"ssm {B}x{H}/{G}x{L}x{d} N {N} {dtype} state {state} lengths {lengths}")
    z = inputs(seed, B, H, G, L, d, N, dtype, state, lengths, fast)
    y, so, dx, ddt, dA, dB, dC, dD, ds = run(z, lengths, D)
    u, r = unit(dtype), share_of(N, d, L)
    f = r + (2.0 ** -16 if dtype == BF else 0.0)  # float32 results
    zero = torch.zeros(H, N, d)
    total = {k: torch.zeros(H, dtype=F64) for k in ("dA", "sA", "dD", "sD")}
    for b in range(B):
        n = L if lengths is None else min(max(lengths[b], 0), L)
        row = [z["x"][b, :, :n], z["dt"][b, :, :n], z["A"], z["Bm"][b, :, :n], z["Cm"][b, :, :n], z["D"] if D else 0 * z["D"],
               zero if z["state"] is None else z["state"][b], z["dy"][b, :, :n], zero if z["dstate"] is None else z["dstate"][b]]
        w, s = exact(row)
        for t in (y, dx, ddt):
            assert not t[b, :, n:].any()
        for t in (dB, dC):
            assert not t[b, :, n:].any()
        close(so[b], w["state"], f * s["state"], f"state[{b}]")
        close(ds[b], w["dh"], f * s["dh"], f"dstate[{b}]")
        if n:
            close(y[b, :, :n], w["y"], (u + r) * s["y"] + u * w["y"].abs(), f"y[{b}]")
            close(dx[b, :, :n], w["dx"], (u + f) * s["dx"] + u * w["dx"].abs(), f"dx[{b}]")
            close(dB[b, :, :n], w["dB"], (u + f) * s["dB"] + u * w["dB"].abs(), f"dB[{b}]")
            close(dC[b, :, :n], w["dC"], (u + f) * s["dC"] + u * w["dC"].abs(), f"dC[{b}]")
            A = z["A"].abs().to(F64)[:, None]
            size = s["ddt"].abs() + 2 * A * s["later"]
            # s["ddt"] carries the sign of A: its parts' sizes are bounded by the later tokens' terms as well
            close(ddt[b, :, :n], w["ddt"], f * size, f"ddt[{b}]")
            total["sA"] += (z["dt"][b, :, :n].to(F64) * s["later"]).sum(1)
        total["dA"] += w["dA"]
        total["dD"] += w["dD"]
        total["sD"] += s["dD"]
    close(dA, total["dA"], 2 * f * total["sA"] + 2.0 ** -24 * total["dA"].abs(), "dA")
    close(dD, total["dD"], f * total["sD"], "dD")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,H,G,L,d,N,state", [
    (1, 1, 1, 1, 32, 8, False),
    (1, 1, 1, 2, 64, 16, True),
    (2, 4, 2, 63, 64, 64, True),
    (2, 3, 1, 64, 32, 24, False),          # N that no tile divides
    (1, 4, 4, 65, 128, 128, True),
    (2, 2, 1, 200, 64, 128, True),
    (1, 6, 2, 130, 128, 64, False),
    (1, 2, 1, 700, 32, 40, True),          # several segments of a sequence
])
def test_forward_and_backward(dtype, B, H, G, L, d, N, state):
    check(B, H, G, L, d, N, dtype, state)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_padded_rows(dtype):
    check(6, 2, 1, 150, 64, 32, dtype, True, lengths=[150, 0, 1, 64, 129, -3])
    check(3, 2, 2, 600, 32, 64, dtype, False, lengths=[600, 65, 333])
    check(2, 2, 1, 150, 64, 32, dtype, False, lengths=[3, 0], D=False)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_decays_of_everything_and_nothing(dtype):
    check(1, 3, 1, 150, 32, 16, dtype, True, fast=True)


def test_no_token():
    """L = 0: the state goes through."""
    z = inputs(3, 2, 2, 1, 0, 64, 32, BF, True)
    y, so = run(z)
    assert y.numel() == 0 and torch.equal(so, z["state"])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,H,G,d,N", [(1, 1, 1, 32, 8), (3, 4, 2, 64, 128), (2, 6, 1, 128, 40), (2, 2, 2, 128, 128), (5, 3, 3, 32, 128)])
def test_step(dtype, B, H, G, d, N):
    bla = _bla()
    z = inputs(7, B, H, G, 1, d, N, dtype, True)
    c = {k: t.cuda() for k, t in z.items()}
    one = [c["x"][:, :, 0].contiguous(), c["dt"][:, :, 0].contiguous(), c["A"], c["Bm"][:, :, 0].contiguous(), c["Cm"][:, :, 0].contiguous()]
    kept, into = c["state"].clone(), torch.empty_like(c["state"])
    y0 = bla.ssm_step(*one, kept, c["D"], state_out=into)
    assert torch.equal(kept, c["state"])
    y = bla.ssm_step(*one, kept, c["D"])   # in place
    assert torch.equal(y, y0) and torch.equal(kept, into)
    u, r = unit(dtype), share_of(N, d, 1)
    for b in range(B):
        w, s = exact([z["x"][b], z["dt"][b], z["A"], z["Bm"][b], z["Cm"][b], z["D"], z["state"][b], z["dy"][b], 0 * z["state"][b]])
        close(into[b].cpu(), w["state"], r * s["state"], f"state[{b}]")
        close(y[b].cpu()[:, None], w["y"], r * s["y"] + u * w["y"].abs(), f"y[{b}]")


def test_prompt_then_tokens():
    """Pieces of a sequence and single tokens after them, in float32."""
    bla = _bla()
    B, H, G, L, d, N = 2, 4, 2, 150, 64, 32
    z = inputs(11, B, H, G, L, d, N, F32, False)
    c = {k: None if t is None else t.cuda() for k, t in z.items()}
    got, state, at = [], None, 0
    cut = lambda t, n: t[:, :, at:at + n].contiguous()  # noqa: E731
    for n in (1, 70, 64):
        y, state = bla.ssm_forward(cut(c["x"], n), cut(c["dt"], n), c["A"], cut(c["Bm"], n), cut(c["Cm"], n), c["D"], state=state)
        got.append(y)
        at += n
    while at < L:
        got.append(bla.ssm_step(*(t[:, :, at].contiguous() for t in (c["x"], c["dt"])), c["A"], c["Bm"][:, :, at].contiguous(),
                                c["Cm"][:, :, at].contiguous(), state, c["D"])[:, :, None])
        at += 1
    got = torch.cat(got, 2).cpu()
    r = share_of(N, d, L) + L * 2.0 ** -23   # a rounding of the state for each single token
    for b in range(B):
        w, s = exact([z["x"][b], z["dt"][b], z["A"], z["Bm"][b], z["Cm"][b], z["D"], torch.zeros(H, N, d), z["dy"][b], torch.zeros(H, N, d)])
        close(got[b], w["y"], r * s["y"], f"y[{b}]")
        close(state[b].cpu(), w["state"], r * s["state"], f"state[{b}]")


def test_backward_against_differences():
    """Directional derivatives of sum(y w) + sum(state v) by central differences of the float32 forward, as for the window."""
    bla = _bla()
    B, H, G, L, d, N = 1, 2, 1, 70, 32, 16
    z = {k: t.cuda() for k, t in inputs(21, B, H, G, L, d, N, F32, True).items()}
    names = ["x", "dt", "A", "Bm", "Cm", "D", "state"]

    def loss(v):
        y, so = bla.ssm_forward(*(v[k] for k in names[:6]), state=v["state"])
        return float((y.double() * z["dy"].double()).sum() + (so.double() * z["dstate"].double()).sum())

    dx, ddt, dA, dB, dC, dD, ds = bla.ssm_backward(*(z[k] for k in names[:5]), z["dy"], z["D"], state=z["state"], dstate=z["dstate"])
    for i, (k, g) in enumerate(zip(names, (dx, ddt, dA, dB, dC, dD, ds))):
        gen = torch.Generator().manual_seed(40 + i)
        step = torch.randn(z[k].shape, generator=gen).cuda() * (z["dt"] * 0.5 if k == "dt" else 1.0)
        h = 2.0 ** -7
        f = [loss({**z, k: z[k] + s * h * step}) for s in (1, -1)]
        num, ana = (f[0] - f[1]) / (2 * h), float((g.double() * step.double()).sum())
        size = float(((g.double() * step.double()) ** 2).sum().sqrt()) + float((g.double() ** 2).sum().sqrt())
        assert abs(num - ana) < 4e-3 * size, (k, num, ana, size)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("L,lengths", [(1930, [1930, 0, 700, 1283]), (1100, [1100, 1099, 321, 64])])
def test_segments(dtype, L, lengths):
    """Rows in four segments whose summaries are taken in parts, some of them past a row's end.  In bf16 a term from an earlier chunk is rounded
    as a weight of the state and with the state: 2u where check() has u; without the state after the call the last segment's weights are
    rounded as well."""
    from ssm_plain import scan
    bla = _bla()
    B, H, G, d, N = 4, 32, 2, 32, 8
    z = inputs(31, B, H, G, L, d, N, dtype, True, lengths)
    c = {k: t.cuda() for k, t in z.items()}
    args = (c["x"], c["dt"], c["A"], c["Bm"], c["Cm"], c["D"])
    kw = dict(state=c["state"], lengths=torch.tensor(lengths, dtype=torch.int32).cuda())
    y, so = bla.ssm_forward(*args, **kw)
    y0, none = bla.ssm_forward(*args, want_state=False, **kw)
    assert none is None
    u, r = unit(dtype), share_of(N, d, L)
    f = r + (2.0 ** -16 if dtype == BF else 0.0)
    for b in range(B):
        n = lengths[b]
        row = [t.to(F64) for t in (z["x"][b, :, :n], z["dt"][b, :, :n], z["A"], z["Bm"][b, :, :n], z["Cm"][b, :, :n], z["D"], z["state"][b])]
        w, end = scan(*row)
        s, size = scan(row[0].abs(), row[1], row[2], *(t.abs() for t in row[3:]))
        close(so[b].cpu(), end, f * size, f"state[{b}]")
        for got in (y, y0):
            assert not got[b, :, n:].any()
            if n:
                close(got[b, :, :n].cpu(), w, (2 * u + r) * s + u * w.abs(), f"y[{b}]")
