"""The selective state space scan token by token in float64, its gradients, and bounds on the kernels' roundings.

The same recurrences on absolute values give the size of every sum's terms.  Rounding a term costs a share of that size: u (the io type's
finfo.eps / 2) where the kernels round an operand to it, and r = (N + d + 400 + 8 chunks) 2^-24 for the float32 sums, the exponentials
(exponents up to 50 in a chunk) and the state carried from chunk to chunk; in bf16 the operands that float32 results
depend on are kept to 2^-17, twice in a product: r + 2^-16.  A gradient through the exponents is a sum over its chunk's later
tokens, so its terms are all of theirs.
"""
import torch

F64 = torch.float64


def scan(x, dt, A, Bm, Cm, D, h, dy=None, dh=None):
    """x [H,n,d], dt [H,n], A, D [H], Bm, Cm [G,n,N], h [H,N,d] (float64).  y and the last state; with dy the gradients as well, and the
    sizes of the sums for ddt's exponents (`chunk`: per token, over the later tokens of its 64-token chunk)."""
    H, n, d = x.shape
    G, N = Bm.shape[0], Bm.shape[-1]
    rep = H // G
    B, C = Bm.repeat_interleave(rep, 0), Cm.repeat_interleave(rep, 0)
    y, states = torch.zeros_like(x), [h]
    for t in range(n):
        h = torch.exp(dt[:, t] * A)[:, None, None] * h + (dt[:, t, None] * B[:, t])[..., None] * x[:, t, None, :]
        y[:, t] = (C[:, t][..., None] * h).sum(1) + D[:, None] * x[:, t]
        states.append(h)
    if dy is None:
        return y, h
    g = dh
    dx, ddt, dB, dC = torch.zeros_like(x), torch.zeros_like(dt), torch.zeros_like(B), torch.zeros_like(C)
    dA = torch.zeros_like(A)
    terms, ends = torch.zeros_like(dt), torch.zeros_like(dt)
    for t in reversed(range(n)):
        if t % 64 == 63 or t == n - 1:
            end = (g * states[t + 1]).sum((1, 2))
        full = g + C[:, t][..., None] * dy[:, t, None, :]
        bg = (B[:, t][..., None] * full).sum(1)
        g = torch.exp(dt[:, t] * A)[:, None, None] * full
        along = (g * states[t]).sum((1, 2))
        dx[:, t] = dt[:, t, None] * bg + D[:, None] * dy[:, t]
        direct = (bg * x[:, t]).sum(-1)
        ddt[:, t] = direct + A * along
        dA += dt[:, t] * along
        dB[:, t] = dt[:, t, None] * (full * x[:, t, None, :]).sum(-1)
        dC[:, t] = (states[t + 1] * dy[:, t, None, :]).sum(-1)
        terms[:, t] = (C[:, t] * dC[:, t]).sum(-1) + dt[:, t] * direct
        ends[:, t] = end
    share = lambda w: w.reshape(G, rep, n, N).sum(1)  # noqa: E731
    later = torch.zeros_like(terms)
    for c in range(0, n, 64):
        later[:, c:c + 64] = terms[:, c:c + 64].flip(1).cumsum(1).flip(1) + ends[:, c:c + 64]
    return {"y": y, "state": states[-1], "dx": dx, "ddt": ddt, "dA": dA, "dB": share(dB), "dC": share(dC), "dD": (x * dy).sum((1, 2)),
            "dh": g, "later": later}


def exact(row):
    """The results of scan() on a row's inputs and the sizes of their terms (absolute values; dt and A as they are)."""
    x, dt, A, Bm, Cm, D, h, dy, dh = (None if t is None else t.to(F64) for t in row)
    want = scan(x, dt, A, Bm, Cm, D, h, dy, dh)
    a = lambda t: None if t is None else t.abs()  # noqa: E731
    size = scan(a(x), dt, A, a(Bm), a(Cm), a(D), a(h), a(dy), a(dh))
    return want, size


def share_of(N, d, n):
    return (N + d + 400 + 8 * ((n + 63) // 64)) * 2.0 ** -24
