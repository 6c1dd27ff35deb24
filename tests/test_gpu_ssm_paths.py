"""The selective scan on shapes of real batches: several heads to a workgroup of the backward pass, and many segments of a sequence.

The recurrence runs in float64 on the GPU over all rows at once (rows are heads of their own; a row's padding is tokens of dt = 0, which leave
the state and every sum as they are).  The bounds are ssm_plain's."""
import pytest
import torch

from ssm_plain import scan, share_of
from test_gpu_parity import _bla, _say
from test_gpu_ssm import inputs
from window_plain import close, unit

pytestmark = pytest.mark.gpu
BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64


def on_gpu(z):
    return {k: None if t is None else t.cuda() for k, t in z.items()}


def folded(c, lengths, back):
    """scan() over all rows, and over absolute values: results [B*H, ...]."""
    B, H, L, d = c["x"].shape
    N = c["Bm"].shape[-1]
    live = torch.arange(L, device="cuda")[None] < torch.tensor([L] * B if lengths is None else lengths, device="cuda")[:, None]
    keep = lambda t: torch.where(live.reshape(B, 1, L, *[1] * (t.dim() - 3)), t.to(F64), 0.0).flatten(0, 1)  # noqa: E731
    zero = torch.zeros(B * H, N, d, dtype=F64, device="cuda")
    state = lambda k: zero if c[k] is None else c[k].to(F64).flatten(0, 1)  # noqa: E731
    row = [keep(c["x"]), keep(c["dt"]), c["A"].to(F64).repeat(B), keep(c["Bm"]), keep(c["Cm"]), c["D"].to(F64).repeat(B), state("state")]
    more = [keep(c["dy"]), state("dstate")] if back else []
    a = lambda t: t.abs()  # noqa: E731
    return scan(*row, *more), scan(a(row[0]), row[1], row[2], *map(a, row[3:] + more)), live


def check_backward(c, lengths):
    bla = _bla()
    B, H, L, d = c["x"].shape
    G, N = c["Bm"].shape[1], c["Bm"].shape[-1]
    dtype = c["x"].dtype
    gl = None if lengths is None else torch.tensor(lengths, dtype=torch.int32).cuda()
    kw = dict(state=c["state"], dstate=c["dstate"], lengths=gl)
    got = [bla.ssm_backward(c["x"], c["dt"], c["A"], c["Bm"], c["Cm"], c["dy"], c["D"], **kw) for _ in range(2)]
    assert all(torch.equal(p, q) for p, q in zip(*got))
    w, s, live = folded(c, lengths, True)
    u, r = unit(dtype), share_of(N, d, L)
    f = r + (2.0 ** -16 if dtype == BF else 0.0)
    A = c["A"].abs().to(F64).repeat(B)[:, None]
    out = dict(zip(("dx", "ddt", "dA", "dB", "dC", "dD", "dh"), got[0]))
    for k, h in (("dx", H), ("dB", G), ("dC", G)):
        t = out[k].flatten(0, 1)
        assert not t[~live.repeat_interleave(h, 0)].any(), k
        close(t, w[k], (u + f) * s[k] + u * w[k].abs(), k)
    close(out["dh"].flatten(0, 1), w["dh"], f * s["dh"], "dstate")
    real = live.repeat_interleave(H, 0)
    assert not out["ddt"].flatten(0, 1)[~real].any()
    close(out["ddt"].flatten(0, 1), torch.where(real, w["ddt"], 0.0), f * (s["ddt"].abs() + 2 * A * s["later"]), "ddt")
    total = lambda t: t.reshape(B, H).sum(0)  # noqa: E731
    dt = torch.where(live[:, None], c["dt"].to(F64), 0.0).flatten(0, 1)
    dA = total(w["dA"])
    close(out["dA"], dA, 2 * f * total((dt * s["later"]).sum(1)) + 2.0 ** -24 * dA.abs(), "dA")
    close(out["dD"], total(w["dD"]), f * total(s["dD"]), "dD")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,H,G,L,d,N,lengths", [
    (64, 6, 2, 200, 32, 16, True),     # 512 groups' chunks: three heads to each workgroup, dB and dC straight to memory
    (32, 10, 2, 200, 64, 40, True),    # 256 of them: five heads as three and two, dB and dC in parts
    (128, 4, 2, 65, 128, 128, False),  # states that do not stay in LDS
    (43, 9, 3, 130, 128, 24, True),
    (60, 4, 1, 520, 32, 128, True),
    (128, 4, 1, 250, 64, 64, False),
])
def test_backward_over_several_heads(dtype, B, H, G, L, d, N, lengths):
    lengths = [max(0, L - 37 * (b % 8)) if b % 5 else [0, 1, 64, L][b // 5 % 4] for b in range(B)] if lengths else None
    _say(f"ssm backward {B}x{H}/{G}x{L}x{d} N {N} {dtype} ragged {lengths is not None}")
    check_backward(on_gpu(inputs(61, B, H, G, L, d, N, dtype, True, lengths)), lengths)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,H,G,L,d,N,lengths", [
    (1, 2, 1, 64 * 40 + 5, 64, 128, None),                       # nine or more segments
    (1, 4, 2, 64 * 140 + 1, 32, 8, None),                        # three batches of the scan over them and more
    (3, 2, 2, 64 * 40, 128, 72, [64 * 40, 64 * 17 + 3, 0]),
    (2, 16, 1, 64 * 16 + 9, 64, 128, [64 * 16 + 9, 64 * 9]),     # four, their summaries in two parts
    (8, 16, 2, 64 * 18, 128, 128, None),
    (2, 3, 1, 64 * 36 + 63, 32, 40, [64 * 36 + 63, 64 * 20 + 1]),
])
def test_segments_that_remember(dtype, B, H, G, L, d, N, lengths):
    """Decays of a few units over the whole sequence, so that what a segment hands on still counts at the end."""
    bla = _bla()
    _say(f"ssm forward {B}x{H}/{G}x{L}x{d} N {N} {dtype} lengths {lengths}")
    z = inputs(71, B, H, G, L, d, N, dtype, True, lengths)
    z["A"] = -torch.rand(H, generator=torch.Generator().manual_seed(72)) * 100.0 / L
    c = on_gpu(z)
    gl = None if lengths is None else torch.tensor(lengths, dtype=torch.int32).cuda()
    y, so = bla.ssm_forward(c["x"], c["dt"], c["A"], c["Bm"], c["Cm"], c["D"], state=c["state"], lengths=gl)
    (w, end), (s, size), live = folded(c, lengths, False)
    u, r = unit(dtype), share_of(N, d, L)
    close(so.flatten(0, 1), end, (r + (2.0 ** -16 if dtype == BF else 0.0)) * size, "state")
    y = y.flatten(0, 1)
    assert not y[~live.repeat_interleave(H, 0)].any()
    # in bf16 a term from an earlier chunk may be rounded as a weight of the state and with the state
    close(y, torch.where(live.repeat_interleave(H, 0)[..., None], w, 0.0), (2 * u + r) * s + u * w.abs(), "y")
