"""Window attention, the short convolution and the selective scan as a model uses them: together, on other streams, captured and replayed,
with shared workspaces, and past 2^32 bytes."""
import math

import pytest
import torch

from ssm_plain import share_of
from test_gpu_parity import _bla, _say
from window_plain import unit

pytestmark = pytest.mark.gpu
BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64


def normal(seed, *shape, dtype=F32, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(dtype)


def rel(a, b):
    return float((a.cpu().to(F64) - b).norm() / b.norm())


def conv64(x, w, b):
    K, L = w.shape[2], x.shape[2]
    e = torch.cat([torch.zeros_like(x[:, :, :K - 1]), x], 2)
    z = b[None, :, None] + sum(e[:, :, j:j + L] * w[None, :, None, :, j] for j in range(K))
    return z * torch.sigmoid(z)


def window64(q, k, v, window, sinks):
    rep, L = q.shape[1] // k.shape[1], q.shape[2]
    k, v = k.repeat_interleave(rep, 1), v.repeat_interleave(rep, 1)
    gap = torch.arange(L)[:, None] - torch.arange(L)[None]
    seen = (gap >= 0) & ((gap < window) | (torch.arange(L)[None] < sinks))
    return torch.softmax((q @ k.transpose(2, 3) / math.sqrt(q.shape[-1])).masked_fill(~seen, -math.inf), -1) @ v


def ssm64(x, dt, A, Bm, Cm, D):
    rep, L = x.shape[1] // Bm.shape[1], x.shape[2]
    Bm, Cm = Bm.repeat_interleave(rep, 1), Cm.repeat_interleave(rep, 1)
    h, y = 0.0, []
    for t in range(L):
        h = torch.exp(dt[:, :, t] * A)[..., None, None] * h + (dt[:, :, t, None] * Bm[:, :, t])[..., None] * x[:, :, t, None, :]
        y.append((Cm[:, :, t][..., None] * h).sum(2) + D[:, None] * x[:, :, t])
    return torch.stack(y, 2)


def test_convolved_window_attention_trains():
    """conv(q), conv(k), conv(v), window attention, and back: outputs and gradients of one loss against float64 autograd.  A stage's
    roundings are a share r of the size of its sums' terms; of n terms of random signs the result is sqrt n below that size, and
    so are n independent roundings, so the relative norms stay below the shares: 4 (r_conv + r_window) over both directions."""
    bla = _bla()
    B, H, Hkv, L, d, K, window, sinks = 2, 4, 2, 150, 64, 4, 40, 3
    heads = (H, Hkv, Hkv)
    xs = [normal(i, B, h, L, d) for i, h in enumerate(heads)]
    ws, bs = [normal(10 + i, h, d, K, std=0.5) for i, h in enumerate(heads)], [normal(20 + i, h, d, std=0.3) for i, h in enumerate(heads)]
    g = normal(30, B, H, L, d)
    leaves = [t.to(F64).requires_grad_() for t in (*xs, *ws, *bs)]
    o64 = window64(*(conv64(leaves[i], leaves[3 + i], leaves[6 + i]) for i in range(3)), window, sinks)
    want = torch.autograd.grad((o64 * g.to(F64)).sum(), leaves)
    c = lambda t: t.cuda()  # noqa: E731
    q, k, v = (bla.conv_forward(c(xs[i]), c(ws[i]), c(bs[i]), want_state=False)[0] for i in range(3))
    o, lse, _, _ = bla.window_forward(q, k, v, window, sinks, want_lse=True)
    grads = bla.window_backward(q, k, v, o, lse, c(g), window, sinks)
    back = [bla.conv_backward(c(xs[i]), c(ws[i]), grads[i], c(bs[i]), want_state_grad=False) for i in range(3)]
    size = float((q.abs() @ k.repeat_interleave(2, 1).abs().transpose(2, 3)).max()) / 8
    r = (K + 8) * 2.0 ** -24 + 2 * (d + 8) * 2.0 ** -24 * size + (window + sinks + 16) * 2.0 ** -24
    assert rel(o, o64.detach()) < 4 * r
    for i in range(3):
        for j, n in ((0, i), (1, 3 + i), (2, 6 + i)):
            assert rel(back[i][j], want[n]) < 4 * r, (i, j)


def test_convolved_scan_trains():
    """conv(x), conv(B), conv(C), scan, and back, likewise."""
    bla = _bla()
    B, H, G, L, d, N, K = 2, 4, 2, 140, 64, 32, 4
    heads, width = (H, G, G), (d, N, N)
    xs = [normal(i, B, h, L, n) for i, (h, n) in enumerate(zip(heads, width))]
    ws = [normal(10 + i, h, n, K, std=0.5) for i, (h, n) in enumerate(zip(heads, width))]
    bs = [normal(20 + i, h, n, std=0.3) for i, (h, n) in enumerate(zip(heads, width))]
    dt, A, D = torch.exp(normal(31, B, H, L) - 3.5), -torch.exp(normal(32, H)), normal(33, H)
    g = normal(34, B, H, L, d)
    leaves = [t.to(F64).requires_grad_() for t in (*xs, *ws, *bs, dt, A, D)]
    y64 = ssm64(conv64(leaves[0], leaves[3], leaves[6]), leaves[9], leaves[10], *(conv64(leaves[i], leaves[3 + i], leaves[6 + i]) for i in (1, 2)),
                leaves[11])
    want = torch.autograd.grad((y64 * g.to(F64)).sum(), leaves)
    c = lambda t: t.cuda()  # noqa: E731
    x, Bm, Cm = (bla.conv_forward(c(xs[i]), c(ws[i]), c(bs[i]), want_state=False)[0] for i in range(3))
    y, _ = bla.ssm_forward(x, c(dt), c(A), Bm, Cm, c(D))
    dx, ddt, dA, dB, dC, dD, _ = bla.ssm_backward(x, c(dt), c(A), Bm, Cm, c(g), c(D), want_state_grad=False)
    back = [bla.conv_backward(c(xs[i]), c(ws[i]), t, c(bs[i]), want_state_grad=False) for i, t in enumerate((dx, dB, dC))]
    r = 4 * (share_of(N, d, L) + (K + 8) * 2.0 ** -24)
    assert rel(y, y64.detach()) < r
    for got, n in ((ddt, 9), (dA, 10), (dD, 11)):
        assert rel(got, want[n]) < r, n
    for i in range(3):
        for j, n in ((0, i), (1, 3 + i), (2, 6 + i)):
            assert rel(back[i][j], want[n]) < r, (i, j)


def state(seed=0, dtype=BF):
    """A small decoding model's buffers: a convolution, a window with its ring, and a scan."""
    B, H, Hkv, d, K, W, S, N = 3, 4, 2, 64, 4, 3000, 4, 32
    c = lambda *s, t=dtype, std=1.0: normal(seed + sum(s), *s, dtype=t, std=std).cuda()  # noqa: E731
    return {"W": W, "S": S, "x": c(B, H, d), "w": c(H, d, K, t=F32), "b": c(H, d, t=F32), "cs": c(B, H, K - 1, d, t=F32), "k": c(B, Hkv, d),
            "v": c(B, Hkv, d, std=2.0), "ck": c(B, Hkv, W + S, d), "cv": c(B, Hkv, W + S, d), "pos": torch.tensor([10, 3003, -1]).cuda(),
            "dt": c(B, H, t=F32).abs() * 0.1, "A": -c(H, t=F32).abs(), "D": c(H, t=F32), "Bm": c(B, 1, N), "Cm": c(B, 1, N),
            "hs": c(B, H, N, d, t=F32)}


def decode(bla, s, room=None):
    q = bla.conv_step(s["x"], s["w"], s["cs"], s["b"])
    o = bla.window_step(q, s["k"], s["v"], s["W"], s["S"], s["ck"], s["cv"], pos=s["pos"], workspace=room)
    y = bla.ssm_step(o, s["dt"], s["A"], s["Bm"], s["Cm"], s["hs"], s["D"])
    s["x"].copy_(y * 0.5)
    s["pos"] += (s["pos"] >= 0).to(torch.int64)
    return y


@pytest.mark.parametrize("dtype", [BF, F32])
def test_captured_decoding(dtype):
    """A captured step, replayed with eager work and synchronisations between, follows the eager steps bit for bit."""
    bla = _bla()
    eager, graph = state(dtype=dtype), state(dtype=dtype)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        decode(bla, state(dtype=dtype))
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = decode(bla, graph)
    for i in range(6):
        want = decode(bla, eager)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
        for k in ("x", "cs", "ck", "cv", "hs", "pos"):
            assert torch.equal(graph[k], eager[k]), (i, k)
        decode(bla, state(7, dtype))  # other work between the replays


def test_captured_prompt_and_backward():
    """Forward and backward calls in one graph, replayed on changed inputs."""
    bla = _bla()
    B, H, Hkv, L, d, W, S, N = 2, 4, 2, 300, 64, 50, 4, 32
    c = lambda i, *s: normal(i, *s, dtype=BF).cuda()  # noqa: E731
    q, k, v, g = c(1, B, H, L, d), c(2, B, Hkv, L, d), c(3, B, Hkv, L, d), c(4, B, H, L, d)
    Bm, Cm, dt, A = c(5, B, 1, L, N), c(6, B, 1, L, N), torch.rand(B, H, L).cuda() * 0.1, -torch.rand(H).cuda()
    w = normal(7, H, d, 4).cuda()

    def step():
        x, st = bla.conv_forward(q, w)
        o, lse, _, _ = bla.window_forward(x, k, v, W, S, want_lse=True)
        y, hs = bla.ssm_forward(o, dt, A, Bm, Cm)
        back = bla.ssm_backward(o, dt, A, Bm, Cm, g)
        dx, dk, dv = bla.window_backward(x, k, v, o, lse, back[0], W, S)
        return [y, hs, st, dk, dv, *back, *bla.conv_backward(q, w, dx)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        q.copy_(c(20 + i, B, H, L, d))
        g.copy_(c(30 + i, B, H, L, d))
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, want)), i


def test_on_another_stream():
    bla = _bla()
    want = decode(bla, state())
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        s = state()
        got = decode(bla, s)
    side.synchronize()
    assert torch.equal(got, want)


def test_on_another_device():
    if torch.cuda.device_count() < 2:
        pytest.skip("one GPU")
    bla = _bla()
    s = {k: v.to("cuda:1") if torch.is_tensor(v) else v for k, v in state().items()}
    want = decode(bla, state())
    assert torch.cuda.current_device() == 0
    assert torch.equal(decode(bla, s).cpu(), want.cpu()) and torch.cuda.current_device() == 0


def test_a_workspace_shared_by_calls():
    """One workspace for calls of every kind, in order on a stream; and one that is too small is replaced."""
    bla = _bla()
    want = decode(bla, state())
    room = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    q, k, v = (normal(i, 1, 2, 20, 64, dtype=BF).cuda() for i in range(3))
    ring = [normal(5 + i, 1, 2, 5004, 64, dtype=BF).cuda() for i in range(2)]
    pos = torch.tensor([7000]).cuda()
    alone = bla.window_forward(q, k, v, 5000, 4, cache_k=ring[0], cache_v=ring[1], pos=pos)[0]
    for size in (room, torch.empty(16, dtype=torch.uint8, device="cuda")):
        a = bla.window_forward(q, k, v, 5000, 4, cache_k=ring[0], cache_v=ring[1], pos=pos, workspace=size)[0]
        assert torch.equal(decode(bla, state(), room=size), want) and torch.equal(a, alone)


def test_tables_end_where_these_calls_write():
    """reuse_tables of the blurry window: a call of these operators in the same workspace ends the record of its tables."""
    bla = _bla()
    B, H, L, d, M, S = 1, 4, 130, 64, 16, 16
    T = [31.0] * H
    q, k, v = (normal(i, B, H, L, d, dtype=BF).cuda() for i in range(3))
    room = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    first = bla.forward(q, k, v, T, M, S, workspace=room)
    ring = [normal(5 + i, 1, 4, 5004, 64, dtype=BF).cuda() for i in range(2)]
    x, w, dt, A, Bm = q, normal(8, H, d, 4).cuda(), torch.rand(B, H, L).cuda(), -torch.rand(H).cuda(), normal(9, B, 1, L, 16, dtype=BF).cuda()
    for call in (lambda: bla.window_step(q[:, :, 0].contiguous(), k[:, :, 0].contiguous(), v[:, :, 0].contiguous(), 5000, 4, *ring, t0=9000, workspace=room),
                 lambda: bla.conv_backward(x, w, x, workspace=room),
                 lambda: bla.ssm_backward(x, dt, A, Bm, Bm, x, workspace=room)):
        call()
        again = bla.forward(q, k, v, T, M, S, workspace=room, reuse_tables=True)
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_refused_tensors():
    bla = _bla()
    q, k = normal(1, 2, 4, 20, 64, dtype=BF).cuda(), normal(2, 2, 2, 20, 64, dtype=BF).cuda()
    bad = [lambda: bla.window_forward(q.transpose(1, 2), k, k, 4),                       # strides
           lambda: bla.window_forward(q, k[:1], k, 4), lambda: bla.window_forward(q, k, k.float(), 4),
           lambda: bla.window_forward(q, k, k, 4, lengths=torch.tensor([3, 4]).cuda()),     # int64 lengths
           lambda: bla.window_forward(q, k, k, 4, cache_k=k), lambda: bla.window_forward(q, k, k, 4, pos=torch.tensor([3, 4])),
           lambda: bla.window_forward(q, k, k, 4, out=q[:1]), lambda: bla.window_step(q[:, :, 0], k[:, :, 0], k[:, :, 0], 4, 0, k, k),
           lambda: bla.conv_forward(q, normal(3, 4, 64, 4)), lambda: bla.conv_forward(q[..., ::2], normal(3, 4, 32, 4).cuda()),
           lambda: bla.conv_step(q[:, :, 0].contiguous(), normal(3, 4, 64, 4).cuda(), k)]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    for f in (lambda: bla.window_forward(q, k, k, 0), lambda: bla.window_forward(q, q[:, :3].contiguous(), q[:, :3].contiguous(), 4),
              lambda: bla.window_forward(q, k, k, 4, out=q), lambda: bla.conv_forward(q, normal(3, 4, 64, 4).cuda(), out=q)):
        with pytest.raises(bla.BlaError):
            f()


def test_a_ring_past_32_bits():
    """4.3 GB of keys: every slot but two holds zeros, and the last head's last slots decide."""
    bla = _bla()
    W, d = 8_400_003, 128
    _say("ring of 2 x 8400003 x 128 bf16")
    ck = torch.zeros(1, 2, W, d, dtype=BF, device="cuda")
    cv = torch.zeros_like(ck)
    q = torch.ones(1, 2, d, dtype=BF, device="cuda")
    k, v = torch.zeros(1, 2, d, dtype=BF, device="cuda"), torch.zeros(1, 2, d, dtype=BF, device="cuda")
    ck[:, :, W - 2], cv[:, :, W - 2] = 2.0, 3.0
    v[:] = 8.0
    o = bla.window_step(q, k, v, W, 0, ck, cv, t0=W - 1)
    e = math.exp(2.0 * d / math.sqrt(d))
    want = (3.0 * e + 8.0) / (e + W - 1)
    torch.cuda.synchronize()
    assert float((o.double() - want).abs().max()) <= 2 * unit(BF) * want * 1.05
    assert torch.equal(cv[:, :, W - 1], v) and torch.equal(ck[:, :, W - 1], k)


def test_tensors_past_32_bits():
    """The last tokens of sequences of 4.3 GB against a short sequence's: a window and a convolution see no further back, and the scan forgets."""
    bla = _bla()
    L, d, n = (1 << 25) + 37, 64, 4096 + 37
    _say("one sequence of 2^25 + 37 tokens")
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.empty(1, 1, L, d, dtype=BF, device="cuda")
    for i in range(0, L, 1 << 22):
        x[:, :, i:i + (1 << 22)] = torch.randn(x[:, :, i:i + (1 << 22)].shape, device="cuda", generator=g)
    tail = x[:, :, L - n:].contiguous()
    w = normal(1, 1, d, 4).cuda()
    y, _ = bla.conv_forward(x, w)
    z, _ = bla.conv_forward(tail, w)
    assert torch.equal(y[:, :, L - 64:], z[:, :, n - 64:])
    o = bla.window_forward(x, x, x, 100, 0, out=y)[0]
    p = bla.window_forward(tail, tail, tail, 100, 0)[0]
    off = (o[:, :, L - 64:].double() - p[:, :, n - 64:].double()).abs()
    assert float((off - 4 * unit(BF) * tail.double().abs().max()).max()) <= 0  # each side off by two units of the values' size
    dt, A = torch.full((1, 1, L), 0.1, device="cuda"), torch.full((1,), -1.0, device="cuda")
    Bm = torch.randn(1, 1, L, 8, device="cuda", generator=g).to(BF)
    y, hs = bla.ssm_forward(x, dt, A, Bm, Bm, out=y)
    z, ht = bla.ssm_forward(tail, dt[:, :, :n].contiguous(), A, Bm[:, :, L - n:].contiguous(), Bm[:, :, L - n:].contiguous())
    size = float(z.double().abs().max())
    assert float((y[:, :, L - 64:].double() - z[:, :, n - 64:].double()).abs().max()) <= 8 * unit(BF) * size
    assert float((hs - ht).abs().max()) <= 1e-5 * float(ht.abs().max())
