"""Sequence operators beside the blurry window: what is measured of them, and their plain forms.

Three operators, each with the call that reads a prompt, its backward pass, and the call that takes one token per row:

  window  softmax attention over the last `window` tokens and the first `sinks` tokens of the sequence; heads share
          keys and values in groups; a row's past lies in a ring of sinks + window slots
          (window_forward, window_backward, window_step)
  conv    the short causal convolution of each channel in front of a sequence operator, with bias and SiLU
          (conv_forward, conv_backward, conv_step)
  ssm     the selective state space scan h_t = exp(dt_t A) h_{t-1} + dt_t B_t x_t^T, y_t = C_t h_t + D x_t of each head
          (ssm_forward, ssm_backward, ssm_step)

The plain forms compute in float32 (running sums of decays in float64) and round once, at the end.
"""
import math

import torch

own = False

F32, F64 = torch.float32, torch.float64
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # a prompt batch of the LM layer of this repository's benchmark (8 x 16 heads x 4096 x 64), four heads to a key head
        {"name": "window prompt", "kind": "window_forward", "dtype": "bf16", "B": 8, "H": 16, "Hkv": 4, "L": 4096, "d": 64,
         "window": 1024, "sinks": 4, "cached": False, "ragged": False},
        # one long document at the long-context width; the window is the 2M - 1 = 255 tokens of M = 128 modes
        {"name": "window long", "kind": "window_forward", "dtype": "bf16", "B": 1, "H": 16, "Hkv": 16, "L": 65536, "d": 128,
         "window": 255, "sinks": 4, "cached": False, "ragged": False},
        # the next pieces of a few prompts in float32, rows of different lengths that continue from their rings
        {"name": "window chunk", "kind": "window_forward", "dtype": "f32", "B": 3, "H": 8, "Hkv": 2, "L": 253, "d": 32,
         "window": 500, "sinks": 3, "cached": True, "ragged": True},
        # the backward pass of a training step on the LM layer's tokens
        {"name": "window training", "kind": "window_backward", "dtype": "bf16", "B": 8, "H": 16, "Hkv": 4, "L": 4096, "d": 64,
         "window": 511, "sinks": 4, "cached": False, "ragged": False},
        # a decode step of a full serving batch (512 rows, as the decode workload), rows at different positions
        {"name": "window step", "kind": "window_step", "dtype": "bf16", "B": 512, "H": 16, "Hkv": 4, "L": 1, "d": 64,
         "window": 1024, "sinks": 4, "cached": True, "ragged": True},
        # a decode step of one conversation: latency
        {"name": "window step alone", "kind": "window_step", "dtype": "bf16", "B": 1, "H": 16, "Hkv": 4, "L": 1, "d": 128,
         "window": 4096, "sinks": 4, "cached": True, "ragged": False},
        # the convolution of the LM layer's queries (or keys, or values) over a prompt batch
        {"name": "conv prompt", "kind": "conv_forward", "dtype": "bf16", "B": 8, "H": 16, "L": 4096, "d": 64, "taps": 4,
         "silu": True, "state": False, "ragged": False},
        # its gradient in a training step
        {"name": "conv training", "kind": "conv_backward", "dtype": "bf16", "B": 8, "H": 16, "L": 4096, "d": 64, "taps": 4,
         "silu": True, "state": False, "ragged": False},
        # a prompt batch of the LM layer's shape through the scan
        {"name": "ssm prompt", "kind": "ssm_forward", "dtype": "bf16", "B": 8, "H": 16, "G": 1, "L": 4096, "d": 64, "N": 128,
         "state": False, "ragged": False},
        # two long rows in float32 that continue from their states, of lengths that no tile divides
        {"name": "ssm long", "kind": "ssm_forward", "dtype": "f32", "B": 2, "H": 8, "G": 2, "L": 16411, "d": 64, "N": 64,
         "state": True, "ragged": True},
        # the backward pass of a training step through the scan
        {"name": "ssm training", "kind": "ssm_backward", "dtype": "bf16", "B": 8, "H": 16, "G": 2, "L": 2048, "d": 64, "N": 64,
         "state": False, "ragged": False},
        # a decode step of a full serving batch: reads and writes every row's state
        {"name": "ssm step", "kind": "ssm_step", "dtype": "bf16", "B": 512, "H": 16, "G": 1, "L": 1, "d": 64, "N": 128,
         "state": True, "ragged": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["window_forward", "window_forward", "window_backward", "window_step", "window_step", "conv_forward",
                       "conv_backward", "conv_step", "ssm_forward", "ssm_forward", "ssm_backward", "ssm_step"])
    c = {"kind": kind, "dtype": rng.choice(["bf16", "bf16", "f32"]), "d": rng.choice([32, 64, 128]), "ragged": rng.random() < 0.4}
    step = kind.endswith("step")
    c["L"] = 1 if step else _log(rng, 1, 65536 if not kind.endswith("backward") else 8192)
    c["H"] = rng.choice([1, 2, 4, 8, 12, 16])
    if kind.endswith("backward"):  # nobody trains on a token, and some of its gradients are nothing but roundings
        c["L"] = max(c["L"], 16)
    c["B"] = _log(rng, 1, 512 if step else 16)
    if kind.startswith("window"):
        c["Hkv"] = rng.choice([g for g in (1, 2, 3, 4, 8, 16) if c["H"] % g == 0])
        c["window"] = _log(rng, 1, 4096)
        c["sinks"] = rng.choice([0, 1, 4, 7, 64])
        c["cached"] = step or (kind == "window_forward" and rng.random() < 0.4)
        if kind == "window_backward":  # a query with one key has no gradient but roundings
            c["window"] = max(c["window"], 8)
    elif kind.startswith("conv"):
        c["taps"] = rng.choice([1, 2, 3, 4, 4, 7])
        c["silu"] = rng.random() < 0.7
        c["state"] = step or rng.random() < 0.5
        c["d"] = rng.choice([32, 64, 128, 8 * _log(rng, 1, 500)])
    else:
        c["G"] = rng.choice([g for g in (1, 2, 4) if c["H"] % g == 0])
        c["N"] = rng.choice([16, 32, 64, 128])
        c["state"] = step or rng.random() < 0.5
    if step and not kind.startswith("window"):
        c["ragged"] = False
    # no dearer than the listed cases of the same kind, by what it computes (float32 products cost sixteen times) and moves
    flops = 8e9 if c["dtype"] == "f32" else 1.2e11
    while (c["L"] > 1 or c["B"] > 1) and (work(c)["flops"] > flops or work(c)["bytes"] > 4.5e8):
        c["B" if c["B"] > 1 else "L"] //= 2
    return c


# ---- what a case's rows look like (the same for every seed) ----

def _lengths(c):
    """Tokens of each row in this call (None: all L)."""
    if not c["ragged"] or c["L"] == 1:
        return None
    L = c["L"]
    return [L if b == 0 else L - (b * 7919) % (L // 2 + 1) for b in range(c["B"])]


def _positions(c):
    """Tokens of each row before this call (None: 0)."""
    if not c.get("cached"):
        return None
    full = c["sinks"] + c["window"]
    if not c["ragged"]:
        return [full + 77] * c["B"]
    return [(b * 6007 + full // 3) % (2 * full + 5) for b in range(c["B"])]


def _pairs(c):
    """Pairs of a query and a visible key, over the rows, for one head."""
    n, W, S = 0, c["window"], c["sinks"]
    pos, lens = _positions(c) or [0] * c["B"], _lengths(c) or [c["L"]] * c["B"]

    def upto(e):  # of the queries at 0 .. e-1
        a = min(e, W)
        inside = a * (a + 1) // 2 + (e - a) * W
        m = max(0, e - W)  # queries with m' = 1 .. m tokens before their window
        s = min(m, S)
        return inside + s * (s + 1) // 2 + (m - s) * S

    for p, l in zip(pos, lens):
        n += upto(p + l) - upto(p)
    return n


def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    B, H, L, d = c["B"], c["H"], c["L"], c["d"]
    toks = sum(_lengths(c) or [L] * B)
    if c["kind"].startswith("window"):
        slots, Hkv = c["sinks"] + c["window"], c["Hkv"]
        pairs = _pairs(c)
        past = sum(min(p, slots) for p in (_positions(c) or [])) * Hkv * d * e * 2
        if c["kind"] == "window_forward":  # q, k, v, the past; o, the sums, the rings where the rows go on
            ring = 2 * B * Hkv * slots * d * e if c["cached"] else 0
            return {"bytes": toks * d * e * 2 * (H + Hkv) + toks * H * 4 + past + ring, "flops": 4 * d * pairs * H}
        if c["kind"] == "window_backward":  # q, k, v, o, dO, the sums; dq, dk, dv
            return {"bytes": toks * d * e * 4 * (H + Hkv) + toks * H * 4, "flops": 10 * d * pairs * H}
        return {"bytes": past + B * d * e * (2 * H + 4 * Hkv), "flops": 4 * d * pairs * H}
    if c["kind"].startswith("conv"):
        n, K = toks * H * d, c["taps"]
        par, st = H * d * (K + 1) * 4, B * H * (K - 1) * d * 4
        if c["kind"] == "conv_forward":
            return {"bytes": 2 * n * e + par + st * (2 if c["state"] else 1), "flops": n * (2 * K + 5)}
        if c["kind"] == "conv_backward":
            return {"bytes": 3 * n * e + 2 * par + st * (3 if c["state"] else 0), "flops": n * (6 * K + 12)}
        return {"bytes": 2 * n * e + par + 2 * st, "flops": n * (2 * K + 5)}
    G, N = c["G"], c["N"]
    st = B * H * N * d * 4
    if c["kind"] == "ssm_step":
        return {"bytes": 2 * st + B * (2 * H * d * e + 4 * H + 2 * G * N * e), "flops": 6 * B * H * N * d}
    if c["kind"] == "ssm_backward":  # 64-token chunks: C B^T, dy x^T, three products with them; six with the states
        return {"bytes": toks * (3 * H * d * e + 8 * H + 4 * G * N * e) + st * (3 if c["state"] else 0),
                "flops": toks * H * (2 * 64 * (3 * N + 2 * d) + 12 * N * d)}
    # 64-token chunks: C B^T, its product with x, the state's reading and its update
    return {"bytes": toks * (2 * H * d * e + 4 * H + 2 * G * N * e) + st * (2 if c["state"] else 1),
            "flops": toks * H * (2 * 64 * N + 2 * 64 * d + 4 * N * d)}


# ---- inputs ----

def prepare(case, seed):
    c = dict(case)
    dev = "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    T = TYPES[c["dtype"]]
    B, H, L, d = c["B"], c["H"], c["L"], c["d"]

    def normal(*shape, std=1.0, dtype=T):
        return (torch.randn(*shape, generator=g, device=dev, dtype=F32) * std).to(dtype)

    def uniform(lo, hi, *shape):
        return torch.rand(*shape, generator=g, device=dev, dtype=F32) * (hi - lo) + lo

    one = c["kind"].endswith("step")
    tok = () if one else (L,)
    lens = _lengths(c)
    s = {"case": c, "lengths": None if lens is None else torch.tensor(lens, dtype=torch.int32, device=dev)}
    if c["kind"].startswith("window"):
        Hkv, slots = c["Hkv"], c["sinks"] + c["window"]
        s["q"], s["k"], s["v"] = normal(B, H, *tok, d, std=1.5), normal(B, Hkv, *tok, d), normal(B, Hkv, *tok, d)
        pos = _positions(c)
        s["pos"] = None if pos is None else torch.tensor(pos, dtype=torch.int64, device=dev)
        if c["cached"]:
            s["cache_k"], s["cache_v"] = normal(B, Hkv, slots, d), normal(B, Hkv, slots, d)
        if c["kind"] == "window_backward":
            s["dO"] = normal(B, H, L, d)
            s["o"], s["lse"] = _window_forward(s)[:2]
        else:
            s["o"] = torch.empty_like(s["q"])
    elif c["kind"].startswith("conv"):
        K = c["taps"]
        s["x"] = normal(B, H, *tok, d)
        s["w"], s["bias"] = uniform(-1, 1, H, d, K) / math.sqrt(K), uniform(-0.5, 0.5, H, d)
        s["state"] = normal(B, H, K - 1, d).to(F32) if c["state"] else None
        if c["kind"] == "conv_backward":
            s["dy"] = normal(B, H, L, d)
            s["dstate"] = normal(B, H, K - 1, d, dtype=F32) if c["state"] else None
        if one:
            s["state_out"] = torch.empty_like(s["state"])
    else:
        G, N = c["G"], c["N"]
        s["x"] = normal(B, H, *tok, d)
        s["dt"] = torch.exp(uniform(math.log(1e-3), math.log(1e-1), B, H, *tok))
        s["A"], s["D"] = -uniform(1, 16, H), uniform(0.5, 1.5, H)
        s["Bm"], s["Cm"] = normal(B, G, *tok, N), normal(B, G, *tok, N)
        s["state"] = normal(B, H, N, d, dtype=F32, std=0.3) if c["state"] else None
        if c["kind"] == "ssm_backward":
            s["dy"] = normal(B, H, L, d)
            s["dstate"] = normal(B, H, N, d, dtype=F32, std=0.3) if c["state"] else None
        if one:
            s["state_out"] = torch.empty_like(s["state"])
    return s


# ---- the framework's calls ----

def _own(s):
    import paper_2606_09862_amd as bla
    c = s["case"]
    kind = c["kind"]
    if kind == "window_forward":
        o, lse, ck, cv = bla.window_forward(s["q"], s["k"], s["v"], c["window"], c["sinks"], lengths=s["lengths"], pos=s["pos"],
                                            cache_k=s.get("cache_k"), cache_v=s.get("cache_v"), want_lse=True,
                                            want_cache=c["cached"])
        return [o, lse] + ([ck, cv] if c["cached"] else [])
    if kind == "window_backward":
        return list(bla.window_backward(s["q"], s["k"], s["v"], s["o"].contiguous(), s["lse"].contiguous(), s["dO"], c["window"], c["sinks"],
                                        lengths=s["lengths"]))
    if kind == "window_step":
        o = bla.window_step(s["q"], s["k"], s["v"], c["window"], c["sinks"], s["cache_k"], s["cache_v"], pos=s["pos"], out=s["o"])
        return [o, s["cache_k"], s["cache_v"]]
    if kind == "conv_forward":
        return list(bla.conv_forward(s["x"], s["w"], s["bias"], silu=c["silu"], state=s["state"], lengths=s["lengths"]))
    if kind == "conv_backward":
        got = bla.conv_backward(s["x"], s["w"], s["dy"], s["bias"], silu=c["silu"], state=s["state"], dstate=s["dstate"],
                                lengths=s["lengths"], want_state_grad=c["state"])
        return list(got) if c["state"] else list(got[:3])
    if kind == "conv_step":
        y = bla.conv_step(s["x"], s["w"], s["state"], s["bias"], silu=c["silu"], state_out=s["state_out"])
        return [y, s["state_out"]]
    if kind == "ssm_forward":
        return list(bla.ssm_forward(s["x"], s["dt"], s["A"], s["Bm"], s["Cm"], s["D"], state=s["state"], lengths=s["lengths"]))
    if kind == "ssm_backward":
        got = bla.ssm_backward(s["x"], s["dt"], s["A"], s["Bm"], s["Cm"], s["dy"], s["D"], state=s["state"], dstate=s["dstate"],
                               lengths=s["lengths"], want_state_grad=c["state"])
        return list(got) if c["state"] else list(got[:6])
    y = bla.ssm_step(s["x"], s["dt"], s["A"], s["Bm"], s["Cm"], s["state"], s["D"], state_out=s["state_out"])
    return [y, s["state_out"]]


# ---- plain forms ----

def _window_parts(s):
    """The band of keys of each block of queries: (queries, keys, values, visible) of the blocks and of the sinks."""
    c = s["case"]
    dev = s["q"].device
    one = c["kind"] == "window_step"
    q, k, v = (x.unsqueeze(2) if one else x for x in (s["q"], s["k"], s["v"]))
    B, H, L, d = q.shape
    Hkv, S = k.shape[1], c["sinks"]
    W = c["window"] if c["cached"] else min(c["window"], L)
    pos = torch.zeros(B, dtype=torch.int64, device=dev) if s["pos"] is None else s["pos"]
    lens = torch.full((B,), L, dtype=torch.int64, device=dev) if s["lengths"] is None else s["lengths"].long()
    # the sequence of keys from W - 1 tokens before the call on, in order of position
    at = pos[:, None] + torch.arange(-(W - 1), L, device=dev)[None]                      # [B, W-1+L]
    real = (at >= S) & (at < (pos + lens)[:, None])
    sat = torch.arange(S, device=dev)[None].expand(B, S)
    sreal = sat < (pos + lens)[:, None]

    def place(new, ring, at, ok):
        old = at < pos[:, None]
        i = (at - pos[:, None]).clamp(0, L - 1)
        got = torch.gather(new.float(), 2, i[:, None, :, None].expand(B, Hkv, -1, d))
        if ring is not None:
            j = torch.where(at < S, at, S + (at - S) % c["window"]).clamp(0, ring.shape[2] - 1)
            past = torch.gather(ring.float(), 2, j[:, None, :, None].expand(B, Hkv, -1, d))
            got = torch.where(old[:, None, :, None], past, got)
        else:
            ok = ok & ~old
        return torch.where(ok[:, None, :, None], got, torch.zeros_like(got)), ok

    rk, rv = s.get("cache_k"), s.get("cache_v")
    ek, ok = place(k, rk, at, real)
    ev, _ = place(v, rv, at, real)
    sk, sok = place(k, rk, sat, sreal)
    sv, _ = place(v, rv, sat, sreal)
    n = min(max(64, min(W, 1024)), L)
    nb = -(-L // n)
    pad = nb * n - L
    group = lambda x: torch.nn.functional.pad(x, (0, 0, 0, pad)).reshape(B, Hkv, H // Hkv, nb, n, d)  # noqa: E731
    blocks = lambda x: torch.nn.functional.pad(x, (0, 0, 0, pad)).unfold(2, n + W - 1, n).transpose(-1, -2)  # noqa: E731
    kat = torch.nn.functional.pad(at, (0, pad), value=-1).unfold(1, n + W - 1, n)        # [B, nb, n+W-1]
    kok = torch.nn.functional.pad(ok, (0, pad)).unfold(1, n + W - 1, n)
    t = torch.arange(nb * n, device=dev)
    qat = (pos[:, None] + t[None]).reshape(B, nb, n)
    qok = (t[None] < lens[:, None]).reshape(B, nb, n)
    seen = kok[:, :, None] & (kat[:, :, None] <= qat[..., None]) & (qat[..., None] - kat[:, :, None] < c["window"]) & qok[..., None]
    sseen = sok[:, None, None] & (sat[:, None, None] <= qat[..., None]) & qok[..., None]
    mask = torch.cat([sseen, seen], -1)[:, None, None]                                  # [B, 1, 1, nb, n, S+n+W-1]
    wide = lambda x: x[:, :, None, None].expand(B, Hkv, 1, nb, S, d)  # noqa: E731
    kk = torch.cat([wide(sk), blocks(ek)[:, :, None]], -2)                             # [B, Hkv, 1, nb, S+n+W-1, d]
    vv = torch.cat([wide(sv), blocks(ev)[:, :, None]], -2)
    return group, q, kk, vv, mask, (n, nb, W, pos, lens)


def _window_scores(s):
    c = s["case"]
    group, q, kk, vv, mask, more = _window_parts(s)
    qq = group(q.float())
    z = torch.matmul(qq, kk.transpose(-1, -2)) * (1.0 / math.sqrt(c["d"]))
    z = torch.where(mask, z, torch.full_like(z, -math.inf))
    top = z.amax(-1, keepdim=True)
    safe = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    p = torch.exp(z - safe)
    total = p.sum(-1, keepdim=True)
    lse = torch.where(total > 0, safe + torch.log(total), torch.full_like(total, -math.inf))
    p = p / torch.where(total > 0, total, torch.ones_like(total))
    return group, qq, kk, vv, p, lse, more


def _rings(s):
    """The rings after the call."""
    c = s["case"]
    one = c["kind"] == "window_step"
    k, v = (x.unsqueeze(2) if one else x for x in (s["k"], s["v"]))
    B, Hkv, L, d = k.shape
    S, W = c["sinks"], c["window"]
    end = s["pos"] + (L if s["lengths"] is None else s["lengths"].long())
    slot = torch.arange(S + W, device=k.device)[None]
    last = end[:, None] - 1
    at = torch.where(slot < S, slot, last - (last - slot) % W)                          # the newest token of each slot
    new = (at >= s["pos"][:, None]) & (at <= last) & (at >= torch.where(slot < S, 0, S))
    i = (at - s["pos"][:, None]).clamp(0, L - 1)[:, None, :, None].expand(B, Hkv, S + W, d)
    take = lambda x, ring: torch.where(new[:, None, :, None], torch.gather(x, 2, i), ring)  # noqa: E731
    return take(k, s["cache_k"]), take(v, s["cache_v"])


def _window_forward(s):
    c = s["case"]
    group, qq, kk, vv, p, lse, (n, nb, W, pos, lens) = _window_scores(s)
    B, L = s["q"].shape[0], c["L"]
    o = torch.matmul(p, vv).reshape(B, c["H"], nb * n, c["d"])[:, :, :L]
    return [o.to(s["q"].dtype), lse.reshape(B, c["H"], nb * n)[:, :, :L].contiguous()]


def _window_backward(s):
    c = s["case"]
    group, qq, kk, vv, p, lse, (n, nb, W, pos, lens) = _window_scores(s)
    B, H, L, d = s["q"].shape
    Hkv, S = c["Hkv"], c["sinks"]
    scale = 1.0 / math.sqrt(d)
    do = group(s["dO"].float())
    do = do * group((torch.arange(L, device=pos.device)[None] < lens[:, None])[:, None, :, None].expand(B, H, L, d).float())
    dp = torch.matmul(do, vv.transpose(-1, -2))
    ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * scale
    del dp
    dq = torch.matmul(ds, kk).reshape(B, H, nb * n, d)[:, :, :L]

    def keys(w, x):  # sums over the heads of a group and over the blocks that hold a key
        got = torch.matmul(w.transpose(-1, -2), x).sum(2)                               # [B, Hkv, nb, S+n+W-1, d]
        first = got[:, :, :, :S].sum(2)
        at = (torch.arange(nb, device=x.device) * n)[:, None] + torch.arange(n + W - 1, device=x.device)[None]
        out = torch.zeros(B, Hkv, nb * n + W - 1, d, device=x.device)
        out.index_add_(2, at.reshape(-1), got[:, :, :, S:].reshape(B, Hkv, -1, d))
        out = out[:, :, W - 1:W - 1 + L].contiguous()
        out[:, :, :S] += first[:, :, :L]
        return out

    dk, dv = keys(ds, qq), keys(p, do)
    return [x.to(s["q"].dtype) for x in (dq, dk, dv)]


def _conv_parts(s):
    c = s["case"]
    one = c["kind"] == "conv_step"
    x = (s["x"].unsqueeze(2) if one else s["x"]).float()
    B, H, L, d = x.shape
    K = c["taps"]
    lens = torch.full((B,), L, dtype=torch.int64, device=x.device) if s["lengths"] is None else s["lengths"].long()
    ok = (torch.arange(L, device=x.device)[None] < lens[:, None])[:, None, :, None]
    past = torch.zeros(B, H, K - 1, d, device=x.device) if s["state"] is None else s["state"]
    ext = torch.cat([past, torch.where(ok, x, torch.zeros_like(x))], 2)
    u = ext.unfold(2, K, 1)                                                             # [B, H, L, d, K]
    z = (u * s["w"][None, :, None]).sum(-1) + s["bias"][None, :, None]
    return ext, u, z, ok, lens


def _conv_forward(s):
    c = s["case"]
    ext, u, z, ok, lens = _conv_parts(s)
    y = z * torch.sigmoid(z) if c["silu"] else z
    y = torch.where(ok, y, torch.zeros_like(y)).to(s["x"].dtype)
    B, H, _, d = ext.shape
    at = lens[:, None] + torch.arange(c["taps"] - 1, device=ext.device)[None]
    state = torch.gather(ext, 2, at[:, None, :, None].expand(B, H, c["taps"] - 1, d))
    return [y.squeeze(2) if c["kind"] == "conv_step" else y, state]


def _conv_backward(s):
    c = s["case"]
    ext, u, z, ok, lens = _conv_parts(s)
    K = c["taps"]
    B, H, E, d = ext.shape
    dz = s["dy"].float()
    if c["silu"]:
        sig = torch.sigmoid(z)
        dz = dz * (sig * (1 + z * (1 - sig)))
    dz = torch.where(ok, dz, torch.zeros_like(dz))
    dw, db = (dz[..., None] * u).sum((0, 2)), dz.sum((0, 2))
    back = torch.nn.functional.pad(dz, (0, 0, K - 1, K - 1)).unfold(2, K, 1)
    dext = (back * s["w"].flip(-1)[None, :, None]).sum(-1)
    if s["dstate"] is not None:
        at = lens[:, None] + torch.arange(K - 1, device=ext.device)[None]
        dext = dext.scatter_add(2, at[:, None, :, None].expand(B, H, K - 1, d), s["dstate"])
    dx = torch.where(ok, dext[:, :, K - 1:], torch.zeros_like(dext[:, :, K - 1:])).to(s["x"].dtype)
    return [dx, dw, db] + ([dext[:, :, :K - 1].contiguous()] if c["state"] else [])


def _ssm_parts(s):
    """64-token chunks: the inputs of each, the exponents of the decays and the states that enter the chunks (and leave the last)."""
    c = s["case"]
    B, H, L, d = s["x"].shape
    G, N, n = c["G"], c["N"], 64
    nb = -(-L // n)
    lens = torch.full((B,), L, dtype=torch.int64, device=s["x"].device) if s["lengths"] is None else s["lengths"].long()
    ok = (torch.arange(L, device=lens.device)[None] < lens[:, None])[:, None]
    pad = nb * n - L
    cut = lambda x: torch.nn.functional.pad(torch.where(ok[..., None], x.float(), 0.0), (0, 0, 0, pad)).reshape(  # noqa: E731
        B, x.shape[1], nb, n, x.shape[-1])
    dt = torch.nn.functional.pad(torch.where(ok, s["dt"], 0.0), (0, pad)).reshape(B, H, nb, n)
    heads = lambda t: t.repeat_interleave(H // G, 1)  # noqa: E731
    x, bm, cm = cut(s["x"]), cut(s["Bm"]), cut(s["Cm"])
    a = torch.cumsum(dt.double() * s["A"].double()[None, :, None, None], -1)              # decay exponents in a chunk
    low = torch.tril(torch.ones(n, n, dtype=torch.bool, device=x.device))
    decay = torch.where(low, torch.exp(torch.where(low, a[..., :, None] - a[..., None, :], 0.0)), 0.0).float()
    total = torch.cumsum(a[..., -1], -1)                                                  # [B, H, nb]
    ends = torch.nn.functional.pad(total, (1, 0))                                         # exponent before chunk 0 .. nb
    past = torch.ones(nb + 1, nb, dtype=torch.bool, device=x.device).tril(-1)
    carry = torch.where(past, torch.exp(torch.where(past, ends[..., :, None] - total[..., None, :], 0.0)), 0.0).float()
    to_end = torch.exp(a[..., -1:] - a).float()
    own_state = torch.matmul((heads(bm) * (to_end * dt)[..., None]).transpose(-1, -2), x)  # [B, H, nb, N, d]
    enter = torch.matmul(carry, own_state.reshape(B, H, nb, N * d)).reshape(B, H, nb + 1, N, d)
    if s["state"] is not None:
        enter = enter + torch.exp(ends).float()[..., None, None] * s["state"][:, :, None]
    return cut, heads, x, bm, cm, dt, a, decay, to_end, ends, enter, (nb, n)


def _ssm_forward(s):
    cut, heads, x, bm, cm, dt, a, decay, to_end, ends, enter, (nb, n) = _ssm_parts(s)
    B, H, L, d = s["x"].shape
    y = torch.matmul(heads(torch.matmul(cm, bm.transpose(-1, -2))) * decay * dt[..., None, :], x)
    y = y + torch.matmul(heads(cm), enter[:, :, :nb]) * torch.exp(a).float()[..., None]
    y = y + s["D"][None, :, None, None, None] * x
    return [y.reshape(B, H, nb * n, d)[:, :, :L].to(s["x"].dtype), enter[:, :, nb].contiguous()]


def _ssm_backward(s):
    cut, heads, x, bm, cm, dt, a, decay, to_end, ends, enter, (nb, n) = _ssm_parts(s)
    B, H, L, d = s["x"].shape
    G, N = s["case"]["G"], s["case"]["N"]
    dy, bh, ch = cut(s["dy"]), heads(bm), heads(cm)
    down = torch.exp(a).float()
    A = s["A"][None, :, None, None]
    # the gradient of the state that leaves each chunk
    own_grad = torch.matmul((ch * down[..., None]).transpose(-1, -2), dy).reshape(B, H, nb, N * d)
    later = torch.ones(nb + 1, nb, dtype=torch.bool, device=x.device).triu(0)
    back = torch.where(later, torch.exp(torch.where(later, ends[..., None, :-1] - ends[..., :, None], 0.0)), 0.0).float()
    g = torch.matmul(back, own_grad).reshape(B, H, nb + 1, N, d)                          # before chunk 0 .. nb
    if s["dstate"] is not None:
        g = g + torch.exp(ends[..., -1:] - ends).float()[..., None, None] * s["dstate"][:, :, None]
    gout, hin = g[:, :, 1:], enter[:, :, :nb]
    cb, yx = heads(torch.matmul(cm, bm.transpose(-1, -2))) * decay, torch.matmul(dy, x.transpose(-1, -2)) * decay
    gb, hy = torch.matmul(bh, gout) * to_end[..., None], torch.matmul(dy, hin.transpose(-1, -2)) * down[..., None]
    gx = torch.matmul(x, gout.transpose(-1, -2)) * to_end[..., None]
    dx = dt[..., None] * (torch.matmul(cb.transpose(-1, -2), dy) + gb) + s["D"][None, :, None, None, None] * dy
    dc = torch.matmul(yx * dt[..., None, :], bh) + hy
    db = dt[..., None] * (torch.matmul(yx.transpose(-1, -2), ch) + gx)
    pair = yx.double() * heads(torch.matmul(cm, bm.transpose(-1, -2))).double()
    late = (gx * bh).double().sum(-1)
    direct = pair.sum(-2) + late
    ds = (pair * dt[..., None, :]).sum(-1) + (hy * ch).double().sum(-1) - dt * direct
    end = (dt * late).sum(-1) + torch.exp(a[..., -1]) * (gout * hin).double().sum((-1, -2))
    da = ds.flip(-1).cumsum(-1).flip(-1) + end[..., None]
    ddt = direct + A * da
    flat = lambda t: t.reshape(t.shape[0], t.shape[1], nb * n, *t.shape[4:])[:, :, :L]  # noqa: E731
    shared = lambda t: flat(t.reshape(B, G, H // G, nb, n, N).sum(2)).to(s["x"].dtype)  # noqa: E731
    ok = torch.arange(L, device=x.device)[None, None] < (L if s["lengths"] is None else s["lengths"].long()[:, None, None])
    got = [flat(dx).to(s["x"].dtype), torch.where(ok, flat(ddt), 0.0).float(), (da * dt).sum((0, 2, 3)).float(), shared(db), shared(dc),
           (dy * x).double().sum((0, 2, 3, 4)).float()]
    return got + ([g[:, :, 0].contiguous()] if s["case"]["state"] else [])


def _ssm_step(s):
    c = s["case"]
    heads = lambda t: t.float().repeat_interleave(c["H"] // c["G"], 1)  # noqa: E731
    x, b, cc = s["x"].float(), heads(s["Bm"]), heads(s["Cm"])
    keep = torch.exp((s["dt"].double() * s["A"].double()[None])).float()
    h = keep[..., None, None] * s["state"] + (s["dt"][..., None] * b)[..., None] * x[..., None, :]
    y = (cc[..., None] * h).sum(-2) + s["D"][None, :, None] * x
    s["state_out"].copy_(h)
    return [y.to(s["x"].dtype), s["state_out"]]


def _window_step(s):
    o = _window_forward({**s, "case": {**s["case"], "L": 1}})[0].squeeze(2)
    ck, cv = _rings(s)
    s["o"].copy_(o)
    s["cache_k"].copy_(ck)
    s["cache_v"].copy_(cv)
    return [s["o"], s["cache_k"], s["cache_v"]]


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    if kind == "window_forward":
        return _window_forward(state) + (list(_rings(state)) if state["case"]["cached"] else [])
    return {"window_backward": _window_backward, "window_step": _window_step, "conv_forward": _conv_forward,
            "conv_backward": _conv_backward, "conv_step": _conv_forward, "ssm_forward": _ssm_forward, "ssm_backward": _ssm_backward,
            "ssm_step": _ssm_step}[kind](state)


# ---- the definitions in 64 bits, row by row and token by token ----

def _exact_window(s):
    c = s["case"]
    one = c["kind"] == "window_step"
    q, k, v = ((x.unsqueeze(2) if one else x).double() for x in (s["q"], s["k"], s["v"]))
    B, H, L, d = q.shape
    Hkv, S, W = c["Hkv"], c["sinks"], c["window"]
    rep = H // Hkv
    back = c["kind"] == "window_backward"
    o, lse = torch.zeros_like(q), torch.full((B, H, L), -math.inf, dtype=F64, device=q.device)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    pos, lens = _positions(c) or [0] * B, _lengths(c) or [L] * B
    size = 1024
    for b in range(B):
        for t in range(0, lens[b], size):
            u = min(lens[b], t + size)
            lo = max(0, pos[b] + t - W + 1)
            at = list(range(min(S, lo))) + list(range(lo, pos[b] + u))
            if not c["cached"]:
                at = [j for j in at if j >= pos[b]]
            old = [j for j in at if j < pos[b]]
            new = torch.tensor([j - pos[b] for j in at if j >= pos[b]], device=q.device)
            ring = torch.tensor([j if j < S else S + (j - S) % W for j in old], dtype=torch.int64, device=q.device)
            kk, vv = (torch.cat([s[n][b].double()[:, ring], x[b][:, new]], 1) if old else x[b][:, new]
                      for n, x in (("cache_k", k), ("cache_v", v)))
            where = torch.tensor(at, device=q.device)
            here = torch.arange(pos[b] + t, pos[b] + u, device=q.device)
            gap = here[:, None] - where[None]
            seen = (gap >= 0) & ((gap < W) | (where[None] < S))
            kh, vh = kk.repeat_interleave(rep, 0), vv.repeat_interleave(rep, 0)
            z = torch.matmul(q[b, :, t:u], kh.transpose(1, 2)) / math.sqrt(d)
            z = z.masked_fill(~seen, -math.inf)
            l = torch.logsumexp(z, -1)
            p = torch.exp(z - l[..., None])
            o[b, :, t:u], lse[b, :, t:u] = torch.matmul(p, vh), l
            if back:
                do = s["dO"][b, :, t:u].double()
                ds = p * (torch.matmul(do, vh.transpose(1, 2)) - (do * o[b, :, t:u]).sum(-1, keepdim=True)) / math.sqrt(d)
                dq[b, :, t:u] = torch.matmul(ds, kh)
                for out, w, y in ((dk, ds, q[b, :, t:u]), (dv, p, do)):
                    out[b].index_add_(1, new, torch.matmul(w.transpose(1, 2), y).reshape(Hkv, rep, len(at), d).sum(1))
    return [dq, dk, dv] if back else [o.squeeze(2) if one else o] + ([] if one else [lse])


def _exact_conv(s):
    c = s["case"]
    one = c["kind"] == "conv_step"
    x = (s["x"].unsqueeze(2) if one else s["x"]).double()
    B, H, L, d = x.shape
    K = c["taps"]
    w, bias = s["w"].double(), s["bias"].double()
    lens = _lengths(c) or [L] * B
    y, dx = torch.zeros_like(x), torch.zeros_like(x)
    state, dstate = (torch.zeros(B, H, K - 1, d, dtype=F64, device=x.device) for _ in range(2))
    dw, db = torch.zeros_like(w), torch.zeros_like(bias)
    for b in range(B):
        n = lens[b]
        past = torch.zeros(H, K - 1, d, dtype=F64, device=x.device) if s["state"] is None else s["state"][b].double()
        line = torch.cat([past, x[b, :, :n]], 1)
        z = bias[:, None].expand(H, n, d).clone()
        for j in range(K):
            z += line[:, j:j + n] * w[:, None, :, j]
        sig = 1 / (1 + torch.exp(-z))
        y[b, :, :n] = z * sig if c["silu"] else z
        state[b] = line[:, n:]
        if c["kind"] == "conv_backward":
            dz = s["dy"][b, :, :n].double()
            dz = dz * (sig + z * sig * (1 - sig)) if c["silu"] else dz
            dline = torch.zeros_like(line)
            for j in range(K):
                dline[:, j:j + n] += dz * w[:, None, :, j]
                dw[:, :, j] += (dz * line[:, j:j + n]).sum(1)
            db += dz.sum(1)
            if s["dstate"] is not None:
                dline[:, n:] += s["dstate"][b].double()
            dx[b, :, :n], dstate[b] = dline[:, K - 1:], dline[:, :K - 1]
    if c["kind"] == "conv_backward":
        return [dx, dw, db] + ([dstate] if c["state"] else [])
    return [y.squeeze(2) if one else y, state]


def _exact_ssm(s):
    c = s["case"]
    one = c["kind"] == "ssm_step"
    x, dt, bm, cm = ((t.unsqueeze(2) if one else t).double() for t in (s["x"], s["dt"], s["Bm"], s["Cm"]))
    B, H, L, d = x.shape
    N, rep = c["N"], H // c["G"]
    A, D = s["A"].double()[None], s["D"].double()[None, :, None]
    lens = torch.tensor(_lengths(c) or [L] * B, device=x.device)[:, None]
    h = torch.zeros(B, H, N, d, dtype=F64, device=x.device) if s["state"] is None else s["state"].double()
    y = torch.zeros_like(x)
    kept = [h]
    for t in range(L):
        go = (t < lens).double()
        step = dt[:, :, t] * go
        h = torch.exp(step * A)[..., None, None] * h
        h = torch.addcmul(h, (step[..., None] * bm[:, :, t].repeat_interleave(rep, 1))[..., None], x[:, :, t, None, :])
        y[:, :, t] = ((cm[:, :, t].repeat_interleave(rep, 1)[..., None] * h).sum(-2) + D * x[:, :, t]) * go[..., None]
        if c["kind"] == "ssm_backward":
            kept.append(h)
    if c["kind"] != "ssm_backward":
        return [y.squeeze(2) if one else y, h]
    g = torch.zeros_like(h) if s["dstate"] is None else s["dstate"].double()
    dx, ddt, db, dc = torch.zeros_like(x), torch.zeros_like(dt), torch.zeros_like(bm), torch.zeros_like(cm)
    dA, dD = torch.zeros(H, dtype=F64, device=x.device), torch.zeros(H, dtype=F64, device=x.device)
    shared = lambda w: w.reshape(B, c["G"], rep, N).sum(2)  # noqa: E731
    for t in reversed(range(L)):
        go = (t < lens).double()
        step = dt[:, :, t] * go
        dy = s["dy"][:, :, t].double() * go[..., None]
        bh, ch, xt = bm[:, :, t].repeat_interleave(rep, 1), cm[:, :, t].repeat_interleave(rep, 1), x[:, :, t] * go[..., None]
        dh = torch.addcmul(g, ch[..., None], dy[..., None, :])
        g = torch.exp(step * A)[..., None, None] * dh
        along = (g * kept[t]).sum((-1, -2))
        bdh = (bh[..., None] * dh).sum(-2)
        dx[:, :, t] = step[..., None] * bdh + D * dy
        ddt[:, :, t] = ((bdh * xt).sum(-1) + A * along) * go
        db[:, :, t] = shared(step[..., None] * (dh * xt[..., None, :]).sum(-1))
        dc[:, :, t] = shared((kept[t + 1] * dy[..., None, :]).sum(-1))
        dA, dD = dA + (step * along).sum(0), dD + (xt * dy).sum((0, 2))
    return [dx, ddt, dA, db, dc, dD] + ([g] if c["state"] else [])


def exact(case, seed):
    c = dict(case)
    kind = c["kind"]
    if kind == "ssm_backward" and c["B"] * c["H"] * c["L"] * c["N"] * c["d"] * 8 > 6e10:  # every token's state
        return None
    s = prepare(c, seed)
    if kind == "window_step":
        return _exact_window(s) + [None, None]
    if kind.startswith("window"):
        return _exact_window(s) + ([None, None] if c.get("cached") else [])
    return _exact_conv(s) if kind.startswith("conv") else _exact_ssm(s)
