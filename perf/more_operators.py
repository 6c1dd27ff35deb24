"""Attention with a learned bias, with a shared prefix, and over a cache of bounded size: what is measured of it, and its plain forms.

Three operators beside window attention, which they extend:

  bias    window attention whose scores carry a learned bias for each head and bucket of distance, with the bias's gradient
          (bias_forward, bias_backward, bias_step)
  prefix  window attention of rows that share a long prefix, every token of which is visible (prefix_forward, prefix_step)
  evict   attention over a cache of `slots` tokens which sums the weight that each token gets from the queries, and gives up the token with the
          least of it (evict_forward: new tokens and the sums; evict_select: the tokens that stay; evict_step: one token)

The plain forms compute in float32 (long sums in float64) and round once, at the end.
"""
import math

import torch

own = False

F32, F64 = torch.float32, torch.float64
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
FAR = 1 << 40  # a window without end


def listed():
    return [
        # a prompt batch at the LM layer's width over its whole causal past, four heads to a key head
        {"name": "bias prompt", "kind": "bias_forward", "dtype": "bf16", "B": 4, "H": 16, "Hkv": 4, "L": 4096, "d": 64, "window": 4096,
         "sinks": 0, "buckets": 32, "far": 128, "cached": False, "ragged": False},
        # the next pieces of a few prompts in float32 that continue from their rings, rows of different lengths, few wide buckets
        {"name": "bias chunk", "kind": "bias_forward", "dtype": "f32", "B": 3, "H": 8, "Hkv": 2, "L": 253, "d": 32, "window": 500,
         "sinks": 3, "buckets": 16, "far": 400, "cached": True, "ragged": True},
        # the backward pass of a training step on the LM layer's heads
        {"name": "bias training", "kind": "bias_backward", "dtype": "bf16", "B": 8, "H": 16, "Hkv": 4, "L": 2048, "d": 64, "window": 2048,
         "sinks": 0, "buckets": 32, "far": 128, "cached": False, "ragged": False},
        # a decode step of a serving batch, rows at different positions
        {"name": "bias step", "kind": "bias_step", "dtype": "bf16", "B": 256, "H": 16, "Hkv": 4, "L": 1, "d": 64, "window": 1024, "sinks": 4,
         "buckets": 32, "far": 512, "cached": True, "ragged": True},
        # a decode step of a serving batch whose rows go on from one long instruction
        {"name": "prefix step", "kind": "prefix_step", "dtype": "bf16", "B": 256, "H": 16, "Hkv": 4, "L": 1, "d": 64, "P": 8192, "G": 1,
         "window": 512, "sinks": 0, "cached": True, "ragged": True},
        # several answers from one document at the long-context width: few rows, a prefix far longer than what they have written
        {"name": "prefix document", "kind": "prefix_step", "dtype": "bf16", "B": 16, "H": 16, "Hkv": 2, "L": 1, "d": 128, "P": 65536, "G": 1,
         "window": 128, "sinks": 0, "cached": True, "ragged": True},
        # a decode step of a small float32 model: latency
        {"name": "prefix small", "kind": "prefix_step", "dtype": "f32", "B": 3, "H": 4, "Hkv": 2, "L": 1, "d": 32, "P": 777, "G": 1,
         "window": 64, "sinks": 4, "cached": True, "ragged": False},
        # questions of different lengths behind two long prefixes
        {"name": "prefix prompt", "kind": "prefix_forward", "dtype": "bf16", "B": 16, "H": 16, "Hkv": 4, "L": 512, "d": 64, "P": 4096, "G": 2,
         "window": 512, "sinks": 0, "cached": False, "ragged": True},
        # a decode step of a full serving batch (512 rows, as the decode workload) over caches of 1024 tokens
        {"name": "evict step", "kind": "evict_step", "dtype": "bf16", "B": 512, "H": 16, "Hkv": 4, "L": 1, "d": 64, "slots": 1024,
         "recent": 64, "cached": True, "ragged": True},
        # a decode step of one conversation: latency
        {"name": "evict step alone", "kind": "evict_step", "dtype": "bf16", "B": 1, "H": 16, "Hkv": 4, "L": 1, "d": 128, "slots": 4096,
         "recent": 512, "cached": True, "ragged": False},
        # two prompts, and the weight that each of their tokens gets
        {"name": "evict prompt", "kind": "evict_forward", "dtype": "bf16", "B": 2, "H": 16, "Hkv": 4, "L": 4096, "d": 64, "slots": 1024,
         "recent": 64, "cached": False, "ragged": False},
        # what stays of the LM layer's prompt batch
        {"name": "evict select", "kind": "evict_select", "dtype": "bf16", "B": 8, "H": 16, "Hkv": 4, "L": 4096, "d": 64, "slots": 1024,
         "recent": 64, "cached": False, "ragged": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["bias_forward", "bias_backward", "bias_step", "prefix_forward", "prefix_step", "prefix_step", "evict_forward",
                       "evict_step", "evict_step", "evict_select"])
    step = kind.endswith("step")
    c = {"kind": kind, "dtype": rng.choice(["bf16", "bf16", "f32"]), "d": rng.choice([32, 64, 128]), "ragged": rng.random() < 0.4,
         "L": 1 if step else _log(rng, 1, 8192), "H": rng.choice([1, 2, 4, 8, 12, 16]), "B": _log(rng, 1, 512 if step else 16)}
    c["Hkv"] = rng.choice([g for g in (1, 2, 3, 4, 8, 16) if c["H"] % g == 0])
    c["cached"] = step or (kind != "bias_backward" and rng.random() < 0.4)
    if kind.startswith("evict"):
        c["slots"] = _log(rng, 2, 4096)
        c["recent"] = rng.randrange(0, c["slots"])
    else:
        c["window"], c["sinks"] = _log(rng, 1, 4096), rng.choice([0, 0, 1, 4, 7, 64])
    if kind.startswith("bias"):
        c["buckets"], c["far"] = rng.choice([2, 8, 16, 32, 64]), _log(rng, 64, 4096)
    if kind.startswith("prefix"):
        c["P"], c["G"] = _log(rng, 1, 65536 if step else 16384), rng.choice([1, 1, 2, 3])
        c["B"] = c["G"] * max(1, c["B"] // c["G"])
    if kind == "bias_backward":  # nobody trains on a token, and a query with one key has no gradient but roundings
        c["L"], c["window"] = max(c["L"], 32), max(c["window"], 16)
    # no dearer than the listed cases, by what it computes (float32 products cost sixteen times), moves, and what its plain form holds
    flops = 8e9 if c["dtype"] == "f32" else 1.2e11
    while work(c)["flops"] > flops or work(c)["bytes"] > 4.5e8 or c["B"] * c["H"] * c["L"] * _span(c) > 1 << 30:
        if c["B"] > c.get("G", 1):
            c["B"] = max(1, c["B"] // c.get("G", 1) // 2) * c.get("G", 1)
        elif c["L"] > 1:
            c["L"] //= 2
        else:
            c["P"] //= 2
    return c


def _span(c):
    """Keys that the plain form holds for a row."""
    if c["kind"].startswith("evict"):
        return c["slots"] + c["L"]
    return c.get("P", 0) + c["sinks"] + (c["window"] if c["cached"] else 0) + c["L"]


def edges_of(buckets, far):
    """The first distance of each bucket but the first: half of them hold one distance each, the others have bounds in geometric progression
    up to `far`: the smallest n with (n / half)^m >= (far / half)^e, in whole numbers."""
    half = buckets // 2
    m = buckets - half
    out = list(range(1, half + 1))
    for e in range(1, m):
        lo, hi = half, max(half, far)
        want = half ** m * max(half, far) ** e
        while lo < hi:
            n = (lo + hi) // 2
            lo, hi = (lo, n) if n ** m * half ** e >= want else (n + 1, hi)
        out.append(lo)
    return tuple(out)


# ---- what a case's rows look like (the same for every seed) ----

def _lengths(c):
    """Tokens of each row in this call (None: all L)."""
    if not c["ragged"] or c["L"] == 1:
        return None
    L = c["L"]
    return [L if b == 0 else L - (b * 7919) % (L // 2 + 1) for b in range(c["B"])]


def _positions(c):
    """Tokens of each row before this call (None: 0)."""
    if not c["cached"]:
        return None
    full = c["slots"] if "slots" in c else c["sinks"] + c["window"]
    if not c["ragged"]:
        return [full + 77] * c["B"]
    return [(b * 6007 + full // 3) % (2 * full + 5) for b in range(c["B"])]


def _prefixes(c):
    """Tokens of each prefix (None: all P)."""
    if c["G"] == 1:
        return None
    return [c["P"] if g == 0 else c["P"] - (g * 7919) % (c["P"] // 2 + 1) for g in range(c["G"])]


def _pairs(c):
    """Pairs of a query and a visible key, over the rows, for one head."""
    n, S = 0, c.get("sinks", 0)
    W = c.get("window", FAR)
    pos, lens = _positions(c) or [0] * c["B"], _lengths(c) or [c["L"]] * c["B"]

    def upto(e):  # of the queries at 0 .. e-1
        a = min(e, W)
        inside = a * (a + 1) // 2 + (e - a) * W
        m = max(0, e - W)  # queries with m' = 1 .. m tokens before their window
        s = min(m, S)
        return inside + s * (s + 1) // 2 + (m - s) * S

    for b, (p, l) in enumerate(zip(pos, lens)):
        if "slots" in c:
            past = min(p, c["slots"])
            past -= 1 if c["kind"] == "evict_step" and past == c["slots"] else 0
            n += l * past + l * (l + 1) // 2
        else:
            n += upto(p + l) - upto(p)
        if "P" in c:
            n += l * (_prefixes(c) or [c["P"]])[b * c["G"] // c["B"]]
    return n


def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    B, H, Hkv, L, d = c["B"], c["H"], c["Hkv"], c["L"], c["d"]
    toks = sum(_lengths(c) or [L] * B)
    full = c["slots"] if "slots" in c else c["sinks"] + c["window"]
    old = sum(min(p, full) for p in (_positions(c) or []))
    past = old * Hkv * d * e * 2
    pairs = _pairs(c)
    if c["kind"] == "evict_select":  # the scores; the tokens that stay, read and written, with their scores and positions
        stay = sum(min(full, n + l) for n, l in zip((min(p, full) for p in _positions(c) or [0] * B), _lengths(c) or [L] * B)) * Hkv
        return {"bytes": (old + toks) * Hkv * 4 + (old * Hkv * 8) + stay * 2 * d * e + B * Hkv * full * (2 * d * e + 12), "flops": (old + toks) * Hkv}
    qkv = toks * d * e * 2 * (H + Hkv)
    if c["kind"] == "bias_backward":  # q, k, v, o, dO, the sums; dq, dk, dv
        return {"bytes": toks * d * e * 4 * (H + Hkv) + toks * H * 4, "flops": 10 * d * pairs * H}
    if c["kind"].startswith("evict"):  # the sums of the past, read and written
        extra = 2 * old * Hkv * 4 + (toks * Hkv * 4 + toks * H * 4 if c["kind"] == "evict_forward" else 2 * old * Hkv * 8)
        return {"bytes": qkv + past + extra, "flops": 4 * d * pairs * H}
    pre = sum(_prefixes(c) or [c["P"]]) * Hkv * d * e * 2 if "P" in c else 0
    ring = 2 * B * Hkv * full * d * e if c["cached"] and c["L"] > 1 else 0
    return {"bytes": qkv + (toks * H * 4 if not c["kind"].endswith("step") else 0) + past + pre + ring, "flops": 4 * d * pairs * H}


# ---- inputs ----

def prepare(case, seed):
    c = dict(case)
    dev = "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    T = TYPES[c["dtype"]]
    B, H, Hkv, L, d = c["B"], c["H"], c["Hkv"], c["L"], c["d"]

    def normal(*shape, std=1.0, dtype=T):
        return (torch.randn(*shape, generator=g, device=dev, dtype=F32) * std).to(dtype)

    def weights(*shape):  # sums of weights so far
        return torch.rand(*shape, generator=g, device=dev, dtype=F32) ** 4 * 8 + 1e-3

    tok = () if c["kind"].endswith("step") else (L,)
    lens, pos = _lengths(c), _positions(c)
    s = {"case": c, "lengths": None if lens is None else torch.tensor(lens, dtype=torch.int32, device=dev),
         "pos": None if pos is None else torch.tensor(pos, dtype=torch.int64, device=dev)}
    s["k"], s["v"] = normal(B, Hkv, *tok, d), normal(B, Hkv, *tok, d)
    if c["kind"] != "evict_select":
        s["q"] = normal(B, H, *tok, d, std=1.5)
        s["o"] = torch.empty_like(s["q"])
    full = c["slots"] if "slots" in c else c["sinks"] + c["window"]
    if c["cached"]:
        s["cache_k"], s["cache_v"] = normal(B, Hkv, full, d), normal(B, Hkv, full, d)
    if "slots" in c and c["cached"]:
        s["score"], s["at"] = weights(B, Hkv, full), _places(c, s["pos"], g)
        if c["kind"] == "evict_step":
            s["score_out"], s["at_out"] = torch.empty_like(s["score"]), torch.empty_like(s["at"])
    if c["kind"] == "evict_select":
        s["score"] = weights(B, Hkv, full + L)
    if "P" in c:
        s["prefix_k"], s["prefix_v"] = normal(c["G"], Hkv, c["P"], d), normal(c["G"], Hkv, c["P"], d)
        n = _prefixes(c)
        s["prefix_lengths"] = None if n is None else torch.tensor(n, dtype=torch.int32, device=dev)
    if "buckets" in c:
        s["bias"], s["edges"] = normal(H, c["buckets"], dtype=F32), edges_of(c["buckets"], c["far"])
    if c["kind"] == "bias_backward":
        s["dO"] = normal(B, H, L, d)
        s["o"], s["lse"] = (x.contiguous() for x in _forward(s)[:2])
    return s


def _places(c, pos, g):
    """The positions of the tokens in each slot: the newest `recent`, and others of the past without order; -1 where there is none."""
    B, Hkv, N, R = c["B"], c["Hkv"], c["slots"], c["recent"]
    dev = pos.device
    slot = torch.arange(N, device=dev)
    pos = pos[:, None, None]
    older = N - R
    step = (pos - R) // older                                                          # 1 and more in a full cache
    spread = slot * step + (torch.rand(B, Hkv, N, generator=g, device=dev) * step).long()
    at = torch.where(slot < older, spread, pos - N + slot)
    at = torch.gather(at, 2, torch.rand(B, Hkv, N, generator=g, device=dev).argsort(-1))
    return torch.where(pos >= N, at, torch.where(slot < pos, slot, -1).expand(B, Hkv, N)).contiguous()


# ---- the framework's calls ----

def _own(s):
    import paper_2606_09862_amd as bla
    c = s["case"]
    kind = c["kind"]
    rows = {"lengths": s["lengths"], "pos": s["pos"]}
    past = {"cache_k": s.get("cache_k"), "cache_v": s.get("cache_v")}
    if kind == "bias_forward":
        o, lse, ck, cv = bla.bias_forward(s["q"], s["k"], s["v"], s["bias"], s["edges"], c["window"], c["sinks"], want_lse=True,
                                          want_cache=c["cached"], **rows, **past)
        return [o, lse] + ([ck, cv] if c["cached"] else [])
    if kind == "bias_backward":
        return list(bla.bias_backward(s["q"], s["k"], s["v"], s["o"], s["lse"], s["dO"], s["bias"], s["edges"], c["window"], c["sinks"],
                                      lengths=s["lengths"]))
    if kind == "bias_step":
        o = bla.bias_step(s["q"], s["k"], s["v"], s["bias"], s["edges"], c["window"], c["sinks"], s["cache_k"], s["cache_v"], pos=s["pos"],
                          out=s["o"])
        return [o, s["cache_k"], s["cache_v"]]
    if kind == "prefix_forward":
        o, lse, ck, cv = bla.prefix_forward(s["q"], s["k"], s["v"], s["prefix_k"], s["prefix_v"], c["window"], c["sinks"],
                                            prefix_lengths=s["prefix_lengths"], want_lse=True, want_cache=c["cached"], **rows, **past)
        return [o, lse] + ([ck, cv] if c["cached"] else [])
    if kind == "prefix_step":
        o = bla.prefix_step(s["q"], s["k"], s["v"], s["prefix_k"], s["prefix_v"], c["window"], c["sinks"], s["cache_k"], s["cache_v"],
                            pos=s["pos"], prefix_lengths=s["prefix_lengths"], out=s["o"])
        return [o, s["cache_k"], s["cache_v"]]
    if kind == "evict_forward":
        return list(bla.evict_forward(s["q"], s["k"], s["v"], c["slots"], score=s.get("score"), want_lse=True, **rows, **past))
    if kind == "evict_select":
        return list(bla.evict_select(s["k"], s["v"], s["score"], c["slots"], c["recent"], at=s.get("at"), **rows, **past))
    o, score, at = bla.evict_step(s["q"], s["k"], s["v"], s["cache_k"], s["cache_v"], s["score"], s["at"], c["recent"], pos=s["pos"],
                                  out=s["o"], score_out=s["score_out"], at_out=s["at_out"])
    return [o, s["cache_k"], s["cache_v"], score, at]


# ---- plain forms ----

def _spans(s):
    """(first position, tokens) of each row in this call, [B]."""
    c = s["case"]
    dev = s["k"].device
    pos = torch.zeros(c["B"], dtype=torch.int64, device=dev) if s["pos"] is None else s["pos"]
    lens = torch.full((c["B"],), c["L"], dtype=torch.int64, device=dev) if s["lengths"] is None else s["lengths"].long()
    return pos, lens


def _new(s, name):
    return s[name].unsqueeze(2) if s["case"]["kind"].endswith("step") else s[name]


def _keys(s):
    """Every key that a row may see: keys and values [B, Hkv, N, d] in float32, positions [B, N] (-1: seen from everywhere), whether it is there."""
    c = s["case"]
    B, Hkv, L, d = c["B"], c["Hkv"], c["L"], c["d"]
    pos, lens = _spans(s)
    dev = pos.device
    ks, vs, ats, oks = [], [], [], []

    def add(k, v, at, ok):
        ks.append(k.float()), vs.append(v.float())
        ats.append(at.expand(B, k.shape[2])), oks.append(ok.expand(B, k.shape[2]))

    if "P" in c:
        row = torch.arange(B, device=dev) * c["G"] // B
        n = torch.full((c["G"],), c["P"], device=dev) if s["prefix_lengths"] is None else s["prefix_lengths"].long()
        add(s["prefix_k"][row], s["prefix_v"][row], torch.full((1, 1), -1, device=dev), torch.arange(c["P"], device=dev)[None] < n[row][:, None])
    if c["cached"] and "slots" in c:
        slot = torch.arange(c["slots"], device=dev)[None]
        add(s["cache_k"], s["cache_v"], torch.full((1, 1), -1, device=dev), slot < pos[:, None])
    elif c["cached"]:
        S, W = c["sinks"], c["window"]
        at = torch.cat([torch.arange(S, device=dev)[None].expand(B, S), pos[:, None] + torch.arange(-(W - 1), 0, device=dev)[None]], 1)
        ok = (at < pos[:, None]) & (at >= 0)
        ok[:, S:] &= at[:, S:] >= S
        slot = torch.where(at < S, at, S + (at - S) % W).clamp(0, S + W - 1)[:, None, :, None].expand(B, Hkv, S + W - 1, d)
        add(torch.gather(s["cache_k"], 2, slot), torch.gather(s["cache_v"], 2, slot), at, ok)
    t = torch.arange(L, device=dev)[None]
    add(_new(s, "k"), _new(s, "v"), pos[:, None] + t, t < lens[:, None])
    return torch.cat(ks, 2), torch.cat(vs, 2), torch.cat(ats, 1), torch.cat(oks, 1)


def _by_distance(s):
    """The bias of each distance up to the last bucket's first, [H, distances], and their buckets."""
    edges = torch.tensor(s["edges"], device=s["bias"].device)
    n = torch.arange(s["edges"][-1] + 1, device=edges.device)
    bucket = (edges[None] <= n[:, None]).sum(1)
    return s["bias"][:, bucket], bucket


def _weights(s, keys):
    """Blocks of queries: (first, last, queries, weights [B, Hkv, grp, n, N], lse [B, H, n], bucket [B, n, N])."""
    c = s["case"]
    k, v, at, ok = keys
    B, H, Hkv, L, d, N = c["B"], c["H"], c["Hkv"], c["L"], c["d"], k.shape[2]
    W, S = c.get("window", FAR), c.get("sinks", 0)
    pos, lens = _spans(s)
    table, buckets = _by_distance(s) if "buckets" in c else (None, None)
    q = _new(s, "q").float().reshape(B, Hkv, H // Hkv, L, d)
    kt = k.transpose(2, 3)[:, :, None]
    n = max(1, min(L, (1 << 27) // (B * H * N)))
    for i in range(0, L, n):
        j = min(L, i + n)
        t = torch.arange(i, j, device=pos.device)[None]
        gap = (pos[:, None] + t)[:, :, None] - at[:, None]                              # [B, n, N]
        seen = (at < 0)[:, None] | ((gap >= 0) & ((gap < W) | (at < S)[:, None]))
        seen = seen & ok[:, None] & (t < lens[:, None])[:, :, None]
        z = torch.matmul(q[:, :, :, i:j], kt) * (1.0 / math.sqrt(d))
        bucket = None
        if table is not None:
            gap = gap.clamp(0, table.shape[1] - 1)
            z = z + table[:, gap].transpose(0, 1).reshape(B, Hkv, H // Hkv, j - i, N)
            bucket = buckets[gap]
        z = torch.where(seen[:, None, None], z, torch.full_like(z, -math.inf))
        top = z.amax(-1, keepdim=True)
        safe = torch.where(torch.isinf(top), torch.zeros_like(top), top)
        p = torch.exp(z - safe)
        total = p.sum(-1, keepdim=True)
        lse = torch.where(total > 0, safe + torch.log(total), torch.full_like(total, -math.inf))
        p = p / torch.where(total > 0, total, torch.ones_like(total))
        yield i, j, q[:, :, :, i:j], p, lse.reshape(B, H, j - i), bucket


def _forward(s):
    """[o, lse], with the sums over the queries of each key's weights [B, Hkv, N] behind them for evict."""
    c = s["case"]
    keys = _keys(s)
    B, H, L, d = c["B"], c["H"], c["L"], c["d"]
    o, lse, got = [], [], 0
    for i, j, _, p, l, _ in _weights(s, keys):
        o.append(torch.matmul(p, keys[1][:, :, None]).reshape(B, H, j - i, d))
        lse.append(l)
        if "slots" in c:
            got = got + p.sum((2, 3), dtype=F64)
    return [torch.cat(o, 2).to(s["q"].dtype), torch.cat(lse, 2), got]


def _rings(s):
    """The rings after the call."""
    c = s["case"]
    k, v = _new(s, "k"), _new(s, "v")
    B, Hkv, L, d = k.shape
    S, W = c["sinks"], c["window"]
    pos, lens = _spans(s)
    last = (pos + lens - 1)[:, None]
    slot = torch.arange(S + W, device=k.device)[None]
    at = torch.where(slot < S, slot, last - (last - slot) % W)                          # the newest token of each slot
    new = (at >= pos[:, None]) & (at <= last) & (at >= torch.where(slot < S, 0, S))
    i = (at - pos[:, None]).clamp(0, L - 1)[:, None, :, None].expand(B, Hkv, S + W, d)
    return [torch.where(new[:, None, :, None], torch.gather(x, 2, i), ring) for x, ring in ((k, s["cache_k"]), (v, s["cache_v"]))]


def _step(s):
    o = _forward(s)[0]
    s["o"].copy_(o.squeeze(2))
    for name, x in zip(("cache_k", "cache_v"), _rings(s)):
        s[name].copy_(x)
    return [s["o"], s["cache_k"], s["cache_v"]]


def _bias_backward(s):
    c = s["case"]
    keys = _keys(s)
    B, H, Hkv, L, d = c["B"], c["H"], c["Hkv"], c["L"], c["d"]
    scale = 1.0 / math.sqrt(d)
    k, v = keys[0][:, :, None], keys[1][:, :, None]
    _, lens = _spans(s)
    real = (torch.arange(L, device=lens.device)[None] < lens[:, None])[:, None, :, None]
    do = torch.where(real, s["dO"].float(), 0.0).reshape(B, Hkv, H // Hkv, L, d)
    dq, dk, dv, db = [], 0, 0, torch.zeros(H, c["buckets"], dtype=F64, device=lens.device)
    for i, j, q, p, _, bucket in _weights(s, keys):
        g = do[:, :, :, i:j]
        dp = torch.matmul(g, v.transpose(-1, -2))
        ds = p * (dp - (p * dp).sum(-1, keepdim=True))
        del dp
        for u in range(c["buckets"]):
            part = torch.where((bucket == u)[:, None, None], ds, 0.0).sum(-1, dtype=F64)
            db[:, u] += part.sum((0, 3)).reshape(H)
        ds = ds * scale
        dq.append(torch.matmul(ds, k).reshape(B, H, j - i, d))
        dk = dk + torch.matmul(ds.transpose(-1, -2), q).sum(2)
        dv = dv + torch.matmul(p.transpose(-1, -2), g).sum(2)
    T = s["q"].dtype
    return [torch.cat(dq, 2).to(T), dk.to(T), dv.to(T), db.float()]


def _evict_forward(s):
    c = s["case"]
    o, lse, got = _forward(s)
    if not c["cached"]:
        got = torch.cat([got.new_zeros(c["B"], c["Hkv"], c["slots"]), got], 2)
    else:
        there = torch.arange(c["slots"], device=got.device)[None] < s["pos"][:, None]
        got[:, :, :c["slots"]] += torch.where(there[:, None], s["score"], 0.0)
    return [o, lse, got.float()]


def _evict_select(s):
    c = s["case"]
    B, Hkv, L, d, N, R = c["B"], c["Hkv"], c["L"], c["d"], c["slots"], c["recent"]
    pos, lens = _spans(s)
    dev = pos.device
    t, slot = torch.arange(L, device=dev), torch.arange(N, device=dev)
    old = s["at"] if c["cached"] else torch.full((B, Hkv, N), -1, device=dev)
    at = torch.cat([old, (pos[:, None, None] + t).expand(B, Hkv, L)], 2)
    there = torch.cat([(slot[None] < pos[:, None]) & bool(c["cached"]), t[None] < lens[:, None]], 1)[:, None]
    late = at >= (pos + lens)[:, None, None] - R
    rank = torch.where(there, torch.where(late, math.inf, s["score"].double()), -math.inf)
    order = torch.sort(rank, dim=-1, descending=True, stable=True)[1][..., :N]
    stay = torch.gather(there.expand(B, Hkv, N + L), 2, order)
    order = torch.where(stay, order, N + L).sort(-1)[0]                                  # those that stay, in the order of their entries
    stay, order = order < N + L, order.clamp(max=N + L - 1)
    pick = lambda x, y: torch.where(stay if x.dim() == 3 else stay[..., None], x, y)  # noqa: E731
    rows = order[..., None].expand(B, Hkv, N, d)
    blank = s["k"].new_zeros(B, Hkv, N, d)
    both = [torch.cat([s["cache_" + n] if c["cached"] else blank, s[n]], 2) for n in ("k", "v")]
    zero = torch.zeros((), dtype=s["k"].dtype, device=dev)
    return [pick(torch.gather(x, 2, rows), zero) for x in both] + [pick(torch.gather(s["score"], 2, order), torch.zeros((), device=dev)),
                                                                    pick(torch.gather(at, 2, order), torch.full((), -1, device=dev))]


def _evict_step(s):
    c = s["case"]
    B, Hkv, N, d = c["B"], c["Hkv"], c["slots"], c["d"]
    pos = s["pos"]
    dev = pos.device
    slot = torch.arange(N, device=dev)
    may = s["at"] < (pos - c["recent"])[:, None, None]
    rank = torch.where(may, s["score"], math.inf)
    least = torch.where(rank == rank.amin(-1, keepdim=True), slot, N).amin(-1)
    mine = torch.where(pos[:, None] < N, pos[:, None], least)                            # [B, Hkv]
    put = mine[..., None, None].expand(B, Hkv, 1, d)
    s["cache_k"].scatter_(2, put, s["k"].unsqueeze(2))
    s["cache_v"].scatter_(2, put, s["v"].unsqueeze(2))
    q = s["q"].float().reshape(B, Hkv, c["H"] // Hkv, d)
    z = torch.matmul(q, s["cache_k"].float().transpose(2, 3)) * (1.0 / math.sqrt(d))
    there = (slot[None] <= pos[:, None])[:, None, None]
    z = torch.where(there, z, torch.full_like(z, -math.inf))
    p = torch.exp(z - z.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    s["o"].copy_(torch.matmul(p, s["cache_v"].float()).reshape(B, c["H"], d))
    here = slot == mine[..., None]
    s["score_out"].copy_(torch.where(here, 0.0, s["score"]) + p.sum(2))
    s["at_out"].copy_(torch.where(here, pos[:, None, None], s["at"]))
    return [s["o"], s["cache_k"], s["cache_v"], s["score_out"], s["at_out"]]


def run(state):
    if own:
        return _own(state)
    c = state["case"]
    if c["kind"] in ("bias_forward", "prefix_forward"):
        return _forward(state)[:2] + (_rings(state) if c["cached"] else [])
    if c["kind"] in ("bias_step", "prefix_step"):
        return _step(state)
    return {"bias_backward": _bias_backward, "evict_forward": _evict_forward, "evict_select": _evict_select,
            "evict_step": _evict_step}[c["kind"]](state)


# ---- the definitions in 64 bits, row by row ----

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "evict_select":
        return _exact_select(s)
    return _exact_evict_step(s) if case["kind"] == "evict_step" else _exact_attention(s)


def _exact_attention(s):
    c = s["case"]
    one = c["kind"].endswith("step")
    q, k, v = ((x.unsqueeze(2) if one else x).double() for x in (s["q"], s["k"], s["v"]))
    B, H, L, d = q.shape
    Hkv, rep, dev = c["Hkv"], H // c["Hkv"], q.device
    W, S, N = c.get("window"), c.get("sinks", 0), c.get("slots", 0)
    pos, lens, pre = _positions(c) or [0] * B, _lengths(c) or [L] * B, _prefixes(c) if "P" in c else None
    o, lse = torch.zeros_like(q), torch.full((B, H, L), -math.inf, dtype=F64, device=dev)
    got = torch.zeros(B, Hkv, N + L, dtype=F64, device=dev)
    back = c["kind"] == "bias_backward"
    dq, dk, dv, db = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v), torch.zeros(H, c.get("buckets", 1), dtype=F64, device=dev)
    rings = [x.clone() for x in (s["cache_k"], s["cache_v"])] if c["cached"] and not N else []
    for b in range(B):
        n, p0 = lens[b], pos[b]
        front_k, front_v, where = [], [], []                                            # what is before the new tokens
        if "P" in c:
            g = b // (B // c["G"])
            m = c["P"] if pre is None else pre[g]
            front_k.append(s["prefix_k"][g, :, :m]), front_v.append(s["prefix_v"][g, :, :m])
            where += [None] * m
        if c["cached"] and N:
            m = min(p0, N)
            front_k.append(s["cache_k"][b, :, :m]), front_v.append(s["cache_v"][b, :, :m])
            where += [None] * m
        elif c["cached"]:
            past = [j for j in range(min(S, p0))] + list(range(max(S, p0 - W + 1, 0), p0))
            at = torch.tensor([j if j < S else S + (j - S) % W for j in past], dtype=torch.int64, device=dev)
            front_k.append(s["cache_k"][b][:, at]), front_v.append(s["cache_v"][b][:, at])
            where += past
        kk = torch.cat([x.double() for x in front_k] + [k[b, :, :n]], 1).repeat_interleave(rep, 0)
        vv = torch.cat([x.double() for x in front_v] + [v[b, :, :n]], 1).repeat_interleave(rep, 0)
        m = len(where)
        every = torch.tensor([x is None for x in where] + [False] * n, device=dev)
        at = torch.tensor([0 if x is None else x for x in where] + list(range(p0, p0 + n)), device=dev)
        if rings:
            for t in range(n):
                j = p0 + t if p0 + t < S else S + (p0 + t - S) % W
                for ring, x in zip(rings, (s["k"], s["v"])):
                    ring[b, :, j] = (x.unsqueeze(2) if one else x)[b, :, t]
        for t in range(0, n, 1024):
            u = min(n, t + 1024)
            gap = torch.arange(p0 + t, p0 + u, device=dev)[:, None] - at[None]
            seen = gap >= 0
            if W is not None:
                seen &= (gap < W) | (at < S)[None]
            seen |= every[None]
            z = torch.matmul(q[b, :, t:u], kk.transpose(1, 2)) / math.sqrt(d)
            if "buckets" in c:
                bucket = torch.bucketize(gap.clamp(min=0), torch.tensor(s["edges"], device=dev), right=True)
                z = z + s["bias"].double()[:, bucket]
            z = z.masked_fill(~seen, -math.inf)
            l = torch.logsumexp(z, -1)
            p = torch.exp(z - l[..., None])
            o[b, :, t:u], lse[b, :, t:u] = torch.matmul(p, vv), l
            if N:
                w = p.sum(1).reshape(Hkv, rep, m + n).sum(1)
                got[b, :, :m] += w[:, :m]
                got[b, :, N:N + n] += w[:, m:]
            if back:
                do = s["dO"][b, :, t:u].double()
                ds = p * (torch.matmul(do, vv.transpose(1, 2)) - (do * o[b, :, t:u]).sum(-1, keepdim=True))
                db.index_add_(1, bucket.reshape(-1), ds.reshape(H, -1))
                ds = ds / math.sqrt(d)
                dq[b, :, t:u] = torch.matmul(ds, kk)
                dk[b, :, :n] += torch.matmul(ds.transpose(1, 2), q[b, :, t:u]).reshape(Hkv, rep, n, d).sum(1)
                dv[b, :, :n] += torch.matmul(p.transpose(1, 2), do).reshape(Hkv, rep, n, d).sum(1)
        if N and c["cached"]:
            got[b, :, :m] += s["score"][b, :, :m].double()
    if back:
        return [dq, dk, dv, db]
    if N:
        return [o, lse, got]
    return [o.squeeze(2)] + rings if one else [o, lse] + rings


def _exact_evict_step(s):
    c = s["case"]
    N, rep = c["slots"], c["H"] // c["Hkv"]
    ck, cv, at = s["cache_k"].clone(), s["cache_v"].clone(), s["at"].clone()
    o, score = torch.zeros(s["q"].shape, dtype=F64, device=ck.device), s["score"].double()
    for b, p in enumerate(_positions(c)):
        if p < N:
            mine = torch.full((c["Hkv"],), p, device=ck.device)
        else:
            mine = torch.argsort(torch.where(at[b] >= p - c["recent"], math.inf, score[b]), stable=True)[:, 0]
        h = torch.arange(c["Hkv"], device=ck.device)
        ck[b, h, mine], cv[b, h, mine], at[b, h, mine], score[b, h, mine] = s["k"][b], s["v"][b], p, 0.0
        n = min(p + 1, N)
        kk, vv = (x[b, :, :n].double().repeat_interleave(rep, 0) for x in (ck, cv))
        w = torch.softmax(torch.matmul(kk, s["q"][b].double()[:, :, None])[..., 0] / math.sqrt(c["d"]), -1)
        o[b] = torch.matmul(w[:, None], vv)[:, 0]
        score[b, :, :n] += w.reshape(c["Hkv"], rep, n).sum(1)
    return [o, ck, cv, score, at]


def _exact_select(s):
    c = s["case"]
    B, Hkv, N, L = c["B"], c["Hkv"], c["slots"], c["L"]
    ck = torch.zeros(B, Hkv, N, c["d"], dtype=s["k"].dtype, device=s["k"].device)
    cv, kept = torch.zeros_like(ck), torch.zeros(B, Hkv, N, dtype=F64, device=ck.device)
    at = torch.full((B, Hkv, N), -1, dtype=torch.int64, device=ck.device)
    pos, lens = _positions(c) or [0] * B, _lengths(c) or [L] * B
    score = s["score"].tolist()
    old = s["at"].tolist() if c["cached"] else None
    for b in range(B):
        n = min(pos[b], N) if c["cached"] else 0
        for h in range(Hkv):
            entries = [(i, old[b][h][i]) for i in range(n)] + [(N + t, pos[b] + t) for t in range(lens[b])]
            rank = sorted(entries, key=lambda x: (x[1] < pos[b] + lens[b] - c["recent"], -score[b][h][x[0]] if x[1] < pos[b] + lens[b] - c["recent"] else 0, x[0]))
            stay = sorted(rank[:N])
            i = torch.tensor([x[0] for x in stay], device=ck.device)
            for out, x, y in ((ck, "cache_k", "k"), (cv, "cache_v", "v")):
                front = s[x][b, h] if c["cached"] else torch.zeros(N, c["d"], dtype=out.dtype, device=out.device)
                out[b, h, :len(stay)] = torch.cat([front, s[y][b, h]], 0)[i]
            kept[b, h, :len(stay)] = s["score"][b, h][i].double()
            at[b, h, :len(stay)] = torch.tensor([x[1] for x in stay], device=ck.device)
    return [ck, cv, kept, at]
