"""Window attention with a learned bias, behind tokens that every query sees, in float64, pair by pair of a full mask: the definition, and bounds
on roundings.

The bounds are window_plain's.  A bias adds its own roundings to a score: the bias in the base-2 domain (two), the score
with it and less the maximum (one each), each by 2^-24 of what is rounded, so
    ds = (d + 8) 2^-24 |scale| max sum_c |q_c k_c| + 4 2^-24 (max |bias| + max |z|).
dbias is a sum of terms that are not rounded to the io type.  A term dS = P (dP - delta) is off by e = r |dS| + P r' and by P times what
delta is off by: the sum over the row of e (and in float32, whose delta comes from the outputs, their rounding).  A wave adds the terms of a lane
one after the other, L + 100 at most, everything beyond is float64:
    |dbias_u - dbias_u*| <= sum over the bucket's pairs of (e + P D_i) + (L + 100) 2^-24 sum of |dS|.
"""
import math

import torch

from window_plain import F64, pairs, slot_of


def bucket_of(n, edges):
    """The number of edges at or below each distance."""
    return sum(((n >= e).to(torch.int64) for e in edges), torch.zeros_like(n))


def row(q, k, v, first, window, sinks, scale, ring_k=None, ring_v=None, front_k=None, front_v=None, bias=None, edges=(), dO=None):
    """One row: q [H,n,d], k, v [Hkv,n,d] (its real tokens only), the ring before it, the tokens that every query sees [Hkv,m,d], the
    bias [H,buckets].  Returns exact results and bounds; "seen_by" is the weight of each key (front, past, new) over the queries and heads of a group."""
    H, n, d = q.shape
    Hkv = k.shape[0]
    rep = H // Hkv
    q, k, v = q.to(F64), k.to(F64), v.to(F64)
    at = torch.arange(first, first + n)
    m = 0 if front_k is None else front_k.shape[1]
    if ring_k is not None:
        past = list(range(min(first, sinks))) + list(range(max(sinks, first - window), first))
        slots = [slot_of(j, window, sinks) for j in past]
        k, v = torch.cat([ring_k.to(F64)[:, slots], k], 1), torch.cat([ring_v.to(F64)[:, slots], v], 1)
        at = torch.cat([torch.tensor(past, dtype=torch.int64), at])
    seen = pairs(q, first, k, at, window, sinks)
    gap = first + torch.arange(n)[:, None] - at[None]
    if m:
        k, v = torch.cat([front_k.to(F64), k], 1), torch.cat([front_v.to(F64), v], 1)
        seen = torch.cat([torch.ones(n, m, dtype=torch.bool), seen], 1)
    kh, vh = k.repeat_interleave(rep, 0), v.repeat_interleave(rep, 0)
    z = q @ kh.transpose(1, 2) * scale
    more = 0.0
    if bias is not None:
        bucket = bucket_of(gap.clamp(min=0), edges)
        b = torch.where(bias < -1e6, -math.inf, bias.to(F64))[:, bucket]  # such pairs have no weight
        z = z + b
        some = z[:, seen]
        more = 4 * 2.0 ** -24 * float(bias[bias >= -1e6].abs().max() if (bias >= -1e6).any() else 0.0)
        more += 4 * 2.0 ** -24 * float(some[torch.isfinite(some)].abs().max() if torch.isfinite(some).any() else 0.0)
    z = z.masked_fill(~seen, -math.inf)
    top = z.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, 0.0)
    P = torch.exp(z - top)
    total = P.sum(-1, keepdim=True)
    lse = (top + torch.log(total))[..., 0]
    P = torch.where(total > 0, P / total, 0.0)
    o = P @ vh
    ds = (d + 8) * 2.0 ** -24 * abs(scale) * float((q.abs() @ kh.abs().transpose(1, 2)).max()) + more
    r = 2 * ds + (k.shape[1] + 16) * 2.0 ** -24
    share = lambda x: x.reshape(Hkv, rep, *x.shape[1:]).sum(1)  # noqa: E731
    got = {"o": o, "lse": lse, "spread": P @ vh.abs(), "r": r, "ds": ds, "seen_by": share(P.sum(1))}
    if dO is not None:
        dO = dO.to(F64)
        delta = (dO * o).sum(-1, keepdim=True)
        dS = P * (dO @ vh.transpose(1, 2) - delta)
        got.update(dq=scale * dS @ kh, dk=scale * share(dS.transpose(1, 2) @ q), dv=share(P.transpose(1, 2) @ dO),
                   dv_spread=share(P.transpose(1, 2) @ dO.abs()))
        rp = (r + (d + 8) * 2.0 ** -24) * (dO.abs() @ vh.abs().transpose(1, 2) + delta.abs())
        lost = (dO * o).abs().sum(-1, keepdim=True)

        def slack(u):
            e = (u + r) * dS.abs() + P * (rp + u * lost)
            return abs(scale) * e @ kh.abs(), abs(scale) * share(e.transpose(1, 2) @ q.abs())
        got["slack"] = slack
        if bias is not None:
            e = r * dS.abs() + P * rp
            off = e.sum(-1, keepdim=True) + 2.0 ** -24 * lost
            term = e + P * off + (n + 100) * 2.0 ** -24 * dS.abs()
            got["db"], got["db_bound"] = (torch.zeros(H, bias.shape[1], dtype=F64).index_add_(1, bucket.reshape(-1), x.reshape(H, -1))
                                          for x in (dS, term))
    return got
