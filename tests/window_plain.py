"""Window attention with sinks in float64, pair by pair of a full mask: the definition, and bounds on roundings.

Bounds.  A value kept in type t is off by at most u = finfo(t).eps / 2 of itself.  The kernels round once to the io type: the weights
(and in the backward pass dS) before their product with the values, and the results; everything else is float32.  A
score is a sum of d products in float32 and is off by at most
    ds = (d + 8) 2^-24 |scale| max sum_c |q_c k_c|,
the weight e^{s - m} by about that much of itself, plus the unit of the exponential, the sum over n keys by n 2^-24.
So with r = 2 ds + (n + 16) 2^-24 (numerator and denominator):
    |o - o*|  <= (u + r) sum_j P_j |v_j| + u |o|
    |dv - dv*| <= (u + r) sum_i P_ij |dO_i| + u |dv|
    |dq - dq*| <= |scale| sum_j e_ij |k_j| + u |dq|,   |dk - dk*| <= |scale| sum_i e_ij |q_i| + u |dk|
    e_ij = (u + r) |dS_ij| + P_ij (r' + u sum_c |dO_ic o_ic|),   r' = (r + (d + 8) 2^-24) (sum_c |dO_ic v_jc| + |delta_i|)
(the last term of e: delta is formed from the rounded outputs).  In float32, u = 2^-24.
"""
import math

import torch

F64 = torch.float64


def unit(dtype):
    return torch.finfo(dtype).eps / 2


def pairs(row_q, first, row_k, at_k, window, sinks):
    """Scores' visibility: queries at first .. first + n - 1, keys at positions at_k."""
    at_q = first + torch.arange(row_q.shape[-2])
    gap = at_q[:, None] - at_k[None]
    return (gap >= 0) & ((gap < window) | (at_k[None] < sinks))


def slot_of(j, window, sinks):
    return j if j < sinks else sinks + (j - sinks) % window


def forward_row(q, k, v, first, window, sinks, scale, ring_k=None, ring_v=None, dO=None):
    """One row: q [H,n,d], k, v [Hkv,n,d] (its real tokens only), the ring before it (or None).
    Returns dicts of exact results and of bounds."""
    H, n, d = q.shape
    Hkv = k.shape[0]
    q, k, v = q.to(F64), k.to(F64), v.to(F64)
    at = torch.arange(first, first + n)
    if ring_k is not None:
        past = list(range(min(first, sinks))) + list(range(max(sinks, first - window), first))
        slots = [slot_of(j, window, sinks) for j in past]
        k = torch.cat([ring_k.to(F64)[:, slots], k], 1)
        v = torch.cat([ring_v.to(F64)[:, slots], v], 1)
        at = torch.cat([torch.tensor(past, dtype=torch.int64), at])
    seen = pairs(q, first, k, at, window, sinks)
    rep = H // Hkv
    kh, vh = k.repeat_interleave(rep, 0), v.repeat_interleave(rep, 0)
    z = (q @ kh.transpose(1, 2) * scale).masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(z, -1)
    P = torch.exp(z - lse[..., None])
    o = P @ vh
    ds = (d + 8) * 2.0 ** -24 * abs(scale) * float((q.abs() @ kh.abs().transpose(1, 2)).max()) if n else 0.0
    r = 2 * ds + (len(at) + 16) * 2.0 ** -24
    got = {"o": o, "lse": lse, "spread": P @ vh.abs(), "r": r, "ds": ds}
    if dO is not None:
        dO = dO.to(F64)
        delta = (dO * o).sum(-1, keepdim=True)
        dS = P * (dO @ vh.transpose(1, 2) - delta)
        share = lambda x: x.reshape(Hkv, rep, *x.shape[1:]).sum(1)  # noqa: E731
        got.update(dq=scale * dS @ kh, dk=scale * share(dS.transpose(1, 2) @ q), dv=share(P.transpose(1, 2) @ dO))
        got["dv_spread"] = share(P.transpose(1, 2) @ dO.abs())

        def slack(u):
            rp = (r + (d + 8) * 2.0 ** -24) * (dO.abs() @ vh.abs().transpose(1, 2) + delta.abs())
            e = (u + r) * dS.abs() + P * (rp + u * (dO * o).abs().sum(-1, keepdim=True))
            return abs(scale) * e @ kh.abs(), abs(scale) * share(e.transpose(1, 2) @ q.abs())
        got["slack"] = slack
    return got


def ring_after(ring, new, first, window, sinks):
    """The ring [Hkv,slots,d] after the tokens new [Hkv,n,d] at positions first ..."""
    ring = ring.clone()
    for i in range(new.shape[1]):
        ring[:, slot_of(first + i, window, sinks)] = new[:, i]
    return ring


def close(got, want, bound, what):
    """Every element within its bound (5 % over it for the second-order terms)."""
    got = got.to(F64)
    off = (got - want).abs() - 1.05 * bound
    assert torch.isfinite(got).all(), f"{what}: not finite"
    assert float(off.max()) <= 0, f"{what}: {float(((got - want).abs() / bound.clamp_min(1e-300)).max()):.3f} of the bound"
