"""Attention with a learned bias, behind a prefix and over a cache of bounded size as a model uses them: together, on other streams, captured and replayed, with
shared workspaces, and past 2^32 bytes."""
import math

import pytest
import torch

from test_gpu_parity import _bla, _say
from test_gpu_sequence_use import conv64, normal, rel
from window_plain import unit

pytestmark = pytest.mark.gpu
BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64
EDGES = (1, 2, 3, 4, 6, 9, 14, 20, 30, 45)


def bias64(q, k, v, bias, window, sinks):
    rep, L = q.shape[1] // k.shape[1], q.shape[2]
    k, v = k.repeat_interleave(rep, 1), v.repeat_interleave(rep, 1)
    gap = torch.arange(L)[:, None] - torch.arange(L)[None]
    seen = (gap >= 0) & ((gap < window) | (torch.arange(L)[None] < sinks))
    bucket = sum((gap >= e).long() for e in EDGES)
    z = q @ k.transpose(2, 3) / math.sqrt(q.shape[-1]) + bias[:, bucket]
    return torch.softmax(z.masked_fill(~seen, -math.inf), -1) @ v


def test_convolved_biased_attention_trains():
    """conv(q), conv(k), conv(v), attention with a learned bias, and back: outputs and gradients of one loss against float64 autograd.  A stage's roundings are a
    share r of the size of its sums' terms; of n terms of random signs the result is sqrt n below that size, and so are n independent roundings, so the
    relative norms stay below the shares: 4 (r_conv + r_attention) over both directions."""
    bla = _bla()
    B, H, Hkv, L, d, K, window, sinks = 2, 4, 2, 150, 64, 4, 150, 0
    heads = (H, Hkv, Hkv)
    xs = [normal(i, B, h, L, d) for i, h in enumerate(heads)]
    ws, bs = [normal(10 + i, h, d, K, std=0.5) for i, h in enumerate(heads)], [normal(20 + i, h, d, std=0.3) for i, h in enumerate(heads)]
    bias, g = normal(29, H, len(EDGES) + 1), normal(30, B, H, L, d)
    leaves = [t.to(F64).requires_grad_() for t in (*xs, *ws, *bs, bias)]
    o64 = bias64(*(conv64(leaves[i], leaves[3 + i], leaves[6 + i]) for i in range(3)), leaves[9], window, sinks)
    want = torch.autograd.grad((o64 * g.to(F64)).sum(), leaves)
    c = lambda t: t.cuda()  # noqa: E731
    q, k, v = (bla.conv_forward(c(xs[i]), c(ws[i]), c(bs[i]), want_state=False)[0] for i in range(3))
    o, lse, _, _ = bla.bias_forward(q, k, v, c(bias), EDGES, window, sinks, want_lse=True)
    *grads, db = bla.bias_backward(q, k, v, o, lse, c(g), c(bias), EDGES, window, sinks)
    back = [bla.conv_backward(c(xs[i]), c(ws[i]), grads[i], c(bs[i]), want_state_grad=False) for i in range(3)]
    size = float((q.abs() @ k.repeat_interleave(2, 1).abs().transpose(2, 3)).max()) / 8 + float(bias.abs().max())
    r = (K + 8) * 2.0 ** -24 + 2 * (d + 12) * 2.0 ** -24 * size + (window + sinks + 16) * 2.0 ** -24
    assert rel(o, o64.detach()) < 4 * r and rel(db, want[9]) < 4 * r
    for i in range(3):
        for j, n in ((0, i), (1, 3 + i), (2, 6 + i)):
            assert rel(back[i][j], want[n]) < 4 * r, (i, j)


def state(seed=0, dtype=BF, B=4):
    """A small decoding model's buffers: a layer with a bias over rings, one behind a prefix, one over a cache of bounded size."""
    H, Hkv, d, W, S, P, N = 4, 2, 64, 500, 4, 1500, 300
    c = lambda *s, t=dtype, std=1.0: normal(seed + sum(s), *s, dtype=t, std=std).cuda()  # noqa: E731
    pos = torch.tensor([10, 503, 700, -1][:B]).cuda()
    at = torch.where(pos[:, None, None] >= N, (pos[:, None, None] - N + torch.arange(N).cuda()), torch.arange(N).cuda()).expand(B, Hkv, N).contiguous()
    return {"W": W, "S": S, "x": c(B, H, d), "k": c(B, Hkv, d), "v": c(B, Hkv, d, std=2.0), "bias": c(H, len(EDGES) + 1, t=F32),
            "bk": c(B, Hkv, W + S, d), "bv": c(B, Hkv, W + S, d), "pk": c(1, Hkv, P, d), "pv": c(1, Hkv, P, d), "rk": c(B, Hkv, W + S, d, std=1.5),
            "rv": c(B, Hkv, W + S, d, std=1.5), "ek": c(B, Hkv, N, d), "ev": c(B, Hkv, N, d), "score": c(B, Hkv, N, t=F32).abs(), "at": at, "pos": pos}


KEPT = ("x", "bk", "bv", "rk", "rv", "ek", "ev", "score", "at", "pos")


def decode(bla, s, room=None):
    more = {"pos": s["pos"], "workspace": room}
    o = bla.bias_step(s["x"], s["k"], s["v"], s["bias"], EDGES, s["W"], s["S"], s["bk"], s["bv"], **more)
    o = bla.prefix_step(o, s["k"], s["v"], s["pk"], s["pv"], s["W"], s["S"], s["rk"], s["rv"], **more)
    o, _, _ = bla.evict_step(o, s["k"], s["v"], s["ek"], s["ev"], s["score"], s["at"], 20, **more)
    s["x"].copy_(o * 0.5)
    s["pos"] += (s["pos"] >= 0).to(torch.int64)
    return o


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
        for k in KEPT:
            assert torch.equal(graph[k], eager[k]), (i, k)
        decode(bla, state(7, dtype))  # other work between the replays


def test_captured_prompt_and_backward():
    """Forward and backward calls, the sums of a prompt's weights and the tokens that stay in one graph, replayed on changed inputs."""
    bla = _bla()
    B, H, Hkv, L, d, N = 2, 4, 2, 300, 64, 100
    c = lambda i, *s, t=BF: normal(i, *s, dtype=t).cuda()  # noqa: E731
    q, k, v, g, bias = c(1, B, H, L, d), c(2, B, Hkv, L, d), c(3, B, Hkv, L, d), c(4, B, H, L, d), c(5, H, len(EDGES) + 1, t=F32)
    pk = c(6, 1, Hkv, 70, d)

    def step():
        o, lse, _, _ = bla.bias_forward(q, k, v, bias, EDGES, L, want_lse=True)
        back = bla.bias_backward(q, k, v, o, lse, g, bias, EDGES, L)
        p, _, ck, cv = bla.prefix_forward(o, k, v, pk, pk, 50, 3, want_cache=True)
        e, _, score = bla.evict_forward(p, k, v, N)
        return [o, *back, p, ck, cv, e, score, *bla.evict_select(k, v, score, N, 10)]

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
        bias.copy_(c(40 + i, H, len(EDGES) + 1, t=F32))
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, want)), i


def test_on_another_stream_and_device():
    bla = _bla()
    want = decode(bla, state())
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        s = state()
        got = decode(bla, s)
        q, k = s["pk"], s["pv"]
        kept = bla.evict_select(q, k, torch.rand(1, 2, 1700, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)), 200)
    side.synchronize()
    assert torch.equal(got, want)
    again = bla.evict_select(q, k, torch.rand(1, 2, 1700, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)), 200)
    assert all(torch.equal(x, y) for x, y in zip(kept, again))
    if torch.cuda.device_count() > 1:
        s = {k: v.to("cuda:1") if torch.is_tensor(v) else v for k, v in state().items()}
        assert torch.equal(decode(bla, s).cpu(), want.cpu()) and torch.cuda.current_device() == 0


def test_a_workspace_shared_by_calls():
    """One workspace for calls of every kind, in order on a stream; one that is too small is replaced; and tables of the blurry window end where these calls write."""
    bla = _bla()
    want = decode(bla, state())
    room = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    B, H, L, d, M, S = 1, 4, 130, 64, 16, 16
    T = [31.0] * H
    q, k, v = (normal(i, B, H, L, d, dtype=BF).cuda() for i in range(3))
    bias = normal(4, H, len(EDGES) + 1).cuda()
    first = bla.forward(q, k, v, T, M, S, workspace=room)
    o, lse, _, _ = bla.bias_forward(q, k, v, bias, EDGES, 60, want_lse=True)
    grads = bla.bias_backward(q, k, v, o, lse, q, bias, EDGES, 60)
    for call in (lambda: decode(bla, state(), room=room), lambda: bla.bias_backward(q, k, v, o, lse, q, bias, EDGES, 60, workspace=room),
                 lambda: bla.evict_forward(q, k, v, 50, workspace=room)):
        got = call()
        again = bla.forward(q, k, v, T, M, S, workspace=room, reuse_tables=True)
        assert all(torch.equal(a, b) for a, b in zip(first, again))
        if isinstance(got, torch.Tensor):
            assert torch.equal(got, want)
        elif len(got) == 4:
            assert all(torch.equal(a, b) for a, b in zip(got, grads))
    assert torch.equal(decode(bla, state(), room=torch.empty(16, dtype=torch.uint8, device="cuda")), want)


def test_refused_tensors():
    bla = _bla()
    q, k = normal(1, 2, 4, 20, 64, dtype=BF).cuda(), normal(2, 2, 2, 20, 64, dtype=BF).cuda()
    b = normal(3, 4, 4).cuda()
    s, at = torch.zeros(2, 2, 30).cuda(), torch.zeros(2, 2, 10, dtype=torch.int64).cuda()
    c10 = k[:, :, :10].contiguous()
    one, kone = q[:, :, 0].contiguous(), k[:, :, 0].contiguous()
    bad = [lambda: bla.bias_forward(q, k, k, b, (1, 2), 4), lambda: bla.bias_forward(q, k, k, b.double(), (1, 2, 3), 4),   # biases and edges
           lambda: bla.bias_forward(q, k, k, b.t(), (1, 2, 3), 4), lambda: bla.bias_forward(q.transpose(1, 2), k, k, b, (1, 2, 3), 4),
           lambda: bla.bias_step(one, kone, kone, b[:3], (1, 2, 3), 4, 0, k, k),
           lambda: bla.prefix_forward(q, k, k, k[0], k[0], 4), lambda: bla.prefix_forward(q, k, k, k.float(), k, 4),
           lambda: bla.prefix_forward(q, k, k, k, k, 4, prefix_lengths=torch.tensor([3, 4]).cuda()),                     # int64
           lambda: bla.prefix_step(one, kone, kone, k[:, :1], k[:, :1], 4, 0, k[:, :, :4].contiguous(), k[:, :, :4].contiguous()),
           lambda: bla.evict_forward(q, k, k, 10, cache_k=c10, cache_v=c10), lambda: bla.evict_select(k, k, s[:, :, :29], 10),
           lambda: bla.evict_select(k, k, s, 10, cache_k=c10, cache_v=c10), lambda: bla.evict_step(one, kone, kone, c10, c10, s, at),
           lambda: bla.evict_step(one, kone, kone, c10, c10.clone(), s[:, :, :10].contiguous(), at.int())]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    for f in (lambda: bla.bias_forward(q, k, k, b, (3, 2, 1), 4), lambda: bla.bias_forward(q, k, k, b, (1, 2, 3), 4, out=q),
              lambda: bla.prefix_forward(q[:1].contiguous(), k[:1].contiguous(), k[:1].contiguous(), k, k, 4),           # two prefixes for one row
              lambda: bla.evict_step(one, kone, kone, c10, c10, s[:, :, :10].contiguous(), at),                          # one tensor as both caches
              lambda: bla.evict_forward(q, k, k, 10, out=q)):
        with pytest.raises(bla.BlaError):
            f()


def test_empty_calls():
    bla = _bla()
    z = lambda *s, t=BF: torch.zeros(*s, dtype=t, device="cuda")  # noqa: E731
    b = z(4, 4, t=F32)
    assert bla.bias_forward(z(2, 4, 0, 64), z(2, 2, 0, 64), z(2, 2, 0, 64), b, (1, 2, 3), 5, want_cache=True)[2].shape == (2, 2, 5, 64)
    assert bla.prefix_forward(z(0, 4, 3, 64), z(0, 2, 3, 64), z(0, 2, 3, 64), z(0, 2, 9, 64), z(0, 2, 9, 64), 5)[0].shape == (0, 4, 3, 64)
    assert bla.prefix_step(z(0, 4, 64), z(0, 2, 64), z(0, 2, 64), z(1, 2, 9, 64), z(1, 2, 9, 64), 5, 0, z(0, 2, 5, 64), z(0, 2, 5, 64)).shape == (0, 4, 64)
    assert bla.evict_forward(z(0, 4, 3, 64), z(0, 2, 3, 64), z(0, 2, 3, 64), 5)[2].shape == (0, 2, 8)
    ck, cv, s, at = bla.evict_select(z(2, 2, 0, 64), z(2, 2, 0, 64), z(2, 2, 5, t=F32), 5)
    assert not ck.any() and not s.any() and bool((at == -1).all())


def test_a_prefix_past_32_bits():
    """4.3 GB of keys: every token but one holds zeros, and that one, near the end of the last head's, decides."""
    bla = _bla()
    P, d = 8_400_003, 128
    _say("prefix of 2 x 8400003 x 128 bf16")
    pk = torch.zeros(1, 2, P, d, dtype=BF, device="cuda")
    pv = torch.zeros_like(pk)
    pk[:, :, P - 2], pv[:, :, P - 2] = 2.0, 3.0
    q, k, v = (torch.full((s[0], s[1], d), x, dtype=BF, device="cuda") for s, x in (((70, 2), 1.0), ((70, 2), 0.0), ((70, 2), 8.0)))
    ring = torch.zeros(70, 2, 4, d, dtype=BF, device="cuda")
    e = math.exp(2.0 * d / math.sqrt(d))
    want = (3.0 * e + 8.0) / (e + P)
    for rows in (1, 70):  # few queries, and tiles
        o = bla.prefix_step(q[:rows], k[:rows], v[:rows], pk, pv, 4, 0, ring[:rows].clone(), ring[:rows].clone())
        f = bla.prefix_forward(q[:rows, :, None], k[:rows, :, None], v[:rows, :, None], pk, pv, 4)[0][:, :, 0]
        torch.cuda.synchronize()
        for x in (o, f):
            assert float((x.double() - want).abs().max()) <= 2 * unit(BF) * want * 1.05, rows


def test_a_cache_past_32_bits():
    """4.3 GB of keys in a cache that is full: the token takes the slot of the least score, the last but one of the last head, and one token decides."""
    bla = _bla()
    N, d = 8_400_003, 128
    _say("cache of 2 x 8400003 x 128 bf16")
    ck = torch.zeros(1, 2, N, d, dtype=BF, device="cuda")
    cv = torch.zeros_like(ck)
    ck[:, :, N - 3], cv[:, :, N - 3] = 2.0, 3.0
    score = torch.ones(1, 2, N, device="cuda")
    score[:, :, N - 2] = 0.5
    at = torch.arange(N, device="cuda").expand(1, 2, N).contiguous()
    q, k, v = (torch.full((1, 2, d), x, dtype=BF, device="cuda") for x in (1.0, 0.0, 8.0))
    o, score, at = bla.evict_step(q, k, v, ck, cv, score, at, recent=1, t0=N)
    e = math.exp(2.0 * d / math.sqrt(d))
    want = (3.0 * e + 8.0) / (e + N - 1)
    torch.cuda.synchronize()
    assert float((o.double() - want).abs().max()) <= 2 * unit(BF) * want * 1.05
    assert torch.equal(cv[:, :, N - 2], v) and bool((at[:, :, N - 2] == N).all()) and bool((at[:, :, N - 1] == N - 1).all())
    assert float((score[:, :, N - 3].double() - 1 - e / (e + N - 1)).abs().max()) < 1e-5 and float((score[:, :, N - 2].double() - 1 / (e + N - 1)).abs().max()) < 1e-9
