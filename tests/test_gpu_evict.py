"""Attention over a cache of bounded size on the GPU against its definition in float64 (past_plain), and the tokens that stay against a sort.

A score is a sum of weights that are each off by r of themselves at most (past_plain's r), added in float32: n queries by one lane after the other, then the
heads: (r + (n + heads + 16) 2^-24) of the sum, and 2^-24 of the score that was there.
"""
import math

import pytest
import torch

from past_plain import row
from test_gpu_parity import _bla, _say
from test_gpu_window import dev, normal
from window_plain import close, unit

pytestmark = pytest.mark.gpu
BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64
ENDLESS = 1 << 40


def weights(seed, *shape):
    g = torch.Generator().manual_seed(seed)
    return torch.rand(*shape, generator=g) ** 4 * 8 + 1e-3


def score_bound(ref, n, rep, before):
    return (ref["r"] + (n + rep + 16) * 2.0 ** -24) * ref["seen_by"] + 2.0 ** -23 * before


def check_forward(B, H, Hkv, L, d, slots, dtype, lengths=None, pos=None, cached=False, seed=0, scale=None, t0=0):
    bla = _bla()
    _say(f"evict forward {B}x{H}/{Hkv}x{L}x{d} slots {slots} {dtype} lengths {lengths} pos {pos} cached {cached}")
    q, k, v = normal(seed, B, H, L, d, dtype=dtype, std=1.5), normal(seed + 1, B, Hkv, L, d, dtype=dtype), normal(seed + 2, B, Hkv, L, d, dtype=dtype)
    ck = cv = sc_in = None
    if cached:  # slots that no token has reached hold NaN
        ck, cv, sc_in = normal(seed + 3, B, Hkv, slots, d, dtype=dtype), normal(seed + 4, B, Hkv, slots, d, dtype=dtype), weights(seed + 5, B, Hkv, slots)
        for b in range(B):
            n = min(max((pos or [t0] * B)[b], 0), slots)
            ck[b, :, n:], cv[b, :, n:], sc_in[b, :, n:] = math.nan, math.nan, math.nan
    if lengths is not None:
        for b in range(B):
            for x in (q, k, v):
                x[b, :, max(0, lengths[b]):] = math.nan
    t = lambda x, ty: None if x is None else torch.tensor(x, dtype=ty)  # noqa: E731
    gq, gk, gv, gck, gcv, gs, gl, gp = dev(q, k, v, ck, cv, sc_in, t(lengths, torch.int32), t(pos, torch.int64))
    o, lse, after = bla.evict_forward(gq, gk, gv, slots, cache_k=gck, cache_v=gcv, score=gs, t0=t0, scale=scale, lengths=gl, pos=gp, want_lse=True)
    o2, none, after2 = bla.evict_forward(gq, gk, gv, slots, cache_k=gck, cache_v=gcv, score=gs, t0=t0, scale=scale, lengths=gl, pos=gp)
    torch.cuda.synchronize()
    assert none is None and torch.equal(o, o2) and torch.equal(after.nan_to_num(-7.0), after2.nan_to_num(-7.0))
    o, lse, after = o.cpu(), lse.cpu(), after.cpu()
    sc = 1 / math.sqrt(d) if scale is None else scale
    u = unit(dtype)
    for b in range(B):
        p = t0 if pos is None else pos[b]
        n = 0 if p < 0 else L if lengths is None else min(max(lengths[b], 0), L)
        m = min(max(p, 0), slots) if cached else 0
        assert not o[b, :, n:].any() and torch.equal(lse[b, :, n:], torch.full_like(lse[b, :, n:], -math.inf))
        assert not after[b, :, slots + n:].any()
        if p < 0 and cached:  # an idle row's scores go through
            assert torch.equal(after[b, :, :slots].nan_to_num(-7.0), sc_in[b].nan_to_num(-7.0))
            continue
        assert not after[b, :, m:slots].any()
        if not n:
            assert m == 0 or torch.equal(after[b, :, :m], sc_in[b, :, :m])
            continue
        ref = row(q[b, :, :n], k[b, :, :n], v[b, :, :n], 0, ENDLESS, 0, sc, front_k=ck[b, :, :m] if m else None, front_v=cv[b, :, :m] if m else None)
        close(o[b, :, :n], ref["o"], (u + ref["r"]) * ref["spread"] + u * ref["o"].abs(), f"o[{b}]")
        close(lse[b, :, :n], ref["lse"], ref["r"] + 2.0 ** -22 * (1 + ref["lse"].abs()), f"lse[{b}]")
        before = torch.cat([sc_in[b, :, :m].to(F64) if m else torch.zeros(Hkv, 0, dtype=F64), torch.zeros(Hkv, n, dtype=F64)], 1)
        got = torch.cat([after[b, :, :m], after[b, :, slots:slots + n]], 1)
        close(got, before + ref["seen_by"], score_bound(ref, n, H // Hkv, before), f"score[{b}]")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,H,Hkv,L,d,slots", [
    (1, 1, 1, 1, 32, 1),
    (2, 4, 2, 65, 64, 7),
    (1, 6, 2, 130, 128, 200),
    (2, 3, 3, 257, 32, 64),
    (1, 20, 1, 333, 64, 100),
    (9, 16, 16, 520, 64, 33),
])
def test_forward(dtype, B, H, Hkv, L, d, slots):
    check_forward(B, H, Hkv, L, d, slots, dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_forward_from_caches(dtype):
    check_forward(6, 4, 2, 70, 64, 40, dtype, pos=[0, 3, 40, 41, 1 << 40, -1], cached=True)
    check_forward(3, 4, 1, 1, 64, 300, dtype, pos=[299, 300, 0], cached=True)
    check_forward(6, 4, 2, 150, 32, 129, dtype, pos=[7, 1000, 128, 129, 130, 5], lengths=[150, 0, 1, 64, 149, -3], cached=True)
    check_forward(2, 2, 1, 5, 64, 4000, dtype, pos=[3990, 9000], cached=True)   # few queries: parts of the keys
    check_forward(2, 2, 2, 33, 128, 64, dtype, t0=90, cached=True, scale=-0.2)
    check_forward(2, 2, 2, 33, 64, 64, dtype, t0=90)                             # positions without a cache


def test_forward_without_tokens():
    """L = 0: the scores go through."""
    bla = _bla()
    z = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    s = weights(1, 2, 1, 5).cuda()
    after = bla.evict_forward(z(2, 2, 0, 32), z(2, 1, 0, 32), z(2, 1, 0, 32), 5, z(2, 1, 5, 32), z(2, 1, 5, 32), s, t0=3)[2].cpu()
    assert torch.equal(after[..., :3], s.cpu()[..., :3]) and not after[..., 3:].any()
    assert not bla.evict_forward(z(2, 2, 0, 32), z(2, 1, 0, 32), z(2, 1, 0, 32), 5)[2].any()


def order_key(x):
    """Scores as numbers, NaN above all."""
    return math.inf if x != x else x, x != x


def stays(entries, score, slots, late):
    """The entries [(index, position)] that stay, in order."""
    sure = [e for e in entries if e[1] >= late]
    rest = sorted((e for e in entries if e[1] < late), key=lambda e: e[0])
    rest.sort(key=lambda e: order_key(score[e[0]]), reverse=True)  # stable also in reverse
    return sorted((sure + rest)[:slots])


def check_select(B, Hkv, L, d, slots, recent, dtype, lengths=None, pos=None, cached=False, seed=0, score=None, at=None):
    bla = _bla()
    _say(f"evict select {B}x{Hkv}x{L}x{d} slots {slots} recent {recent} {dtype} lengths {lengths} pos {pos} cached {cached}")
    k, v = normal(seed, B, Hkv, L, d, dtype=dtype), normal(seed + 1, B, Hkv, L, d, dtype=dtype)
    score = weights(seed + 2, B, Hkv, slots + L) if score is None else score
    ck = cv = None
    if cached:
        ck, cv = normal(seed + 3, B, Hkv, slots, d, dtype=dtype), normal(seed + 4, B, Hkv, slots, d, dtype=dtype)
        if at is None:
            g = torch.Generator().manual_seed(seed + 5)
            at = torch.full((B, Hkv, slots), -1)
            for b in range(B):
                m = min(max(pos[b], 0), slots)
                for h in range(Hkv):
                    old = torch.randperm(min(max(pos[b], 0), 10 ** 6), generator=g)[:m]
                    new = torch.arange(pos[b] - min(recent, m), pos[b])   # the newest are always there
                    old = old[old < pos[b] - len(new)][: m - len(new)]
                    more = torch.tensor([x for x in range(max(pos[b], 0)) if x not in set(old.tolist()) | set(new.tolist())][: m - len(new) - len(old)], dtype=torch.int64)
                    every = torch.cat([old, new, more])
                    at[b, h, :m] = every[torch.randperm(m, generator=g)]
    t = lambda x, ty: None if x is None else torch.tensor(x, dtype=ty)  # noqa: E731
    gk, gv, gs, gck, gcv, ga, gl, gp = dev(k, v, score, ck, cv, at if cached else None, t(lengths, torch.int32), t(pos, torch.int64))
    got = bla.evict_select(gk, gv, gs, slots, recent, cache_k=gck, cache_v=gcv, at=ga, lengths=gl, pos=gp)
    torch.cuda.synchronize()
    ok, ov, os, oa = (x.cpu() for x in got)
    for b in range(B):
        p = 0 if pos is None else pos[b]
        n = 0 if p < 0 else L if lengths is None else min(max(lengths[b], 0), L)
        m = min(max(p, 0), slots) if cached else 0
        for h in range(Hkv):
            if p < 0:
                entries = [(i, int(at[b, h, i])) for i in range(slots)] if cached else []
                keep = entries
            else:
                entries = [(i, int(at[b, h, i])) for i in range(m)] + [(slots + i, p + i) for i in range(n)]
                keep = stays(entries, score[b, h].tolist(), slots, p + n - recent)
            i = torch.tensor([e[0] for e in keep], dtype=torch.int64)
            c = len(keep)
            for out, old, new in ((ok, ck, k), (ov, cv, v)):
                every = torch.cat([old[b, h] if cached else torch.zeros(slots, d, dtype=dtype), new[b, h]], 0)
                assert torch.equal(out[b, h, :c], every[i]) and not out[b, h, c:].any(), (b, h)
            assert torch.equal(os[b, h, :c].nan_to_num(-7.0), score[b, h][i].nan_to_num(-7.0)) and not os[b, h, c:].any(), (b, h)
            assert oa[b, h].tolist() == [e[1] for e in keep] + [-1] * (slots - c), (b, h)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_select(dtype):
    check_select(1, 1, 1, 32, 1, 0, dtype)
    check_select(2, 2, 100, 64, 200, 5, dtype)                                       # everything stays
    check_select(2, 2, 300, 64, 200, 0, dtype)
    check_select(2, 3, 300, 128, 77, 76, dtype, lengths=[300, 78])
    check_select(5, 2, 70, 32, 50, 9, dtype, lengths=[70, 0, 1, 49, 51])
    check_select(6, 2, 70, 64, 50, 9, dtype, pos=[0, 3, 50, 51, 400, -1], cached=True)
    check_select(4, 1, 1, 64, 33, 32, dtype, pos=[32, 33, 34, 1000], cached=True)
    check_select(3, 1, 0, 32, 20, 4, dtype, pos=[5, 20, 90], cached=True)             # no new tokens
    check_select(2, 1, 10, 32, 20, 4, dtype, pos=[5, -3])                             # positions without a cache


def test_select_many():
    """More entries than LDS holds, and scores that differ in their last bits alone."""
    check_select(1, 2, 30011, 32, 1000, 17, BF)
    base = torch.full((1, 1, 30000 + 555), 1.0)
    g = torch.Generator().manual_seed(3)
    base += torch.randint(0, 4000, base.shape, generator=g) * 2.0 ** -23
    check_select(1, 1, 30000, 32, 555, 3, BF, score=base)


def test_select_at_a_step():
    """As many large scores as slots, told from the others by the first bits of their keys, by the next, or by the last; and one more or less."""
    for low in (1.0, 2.0 - 2.0 ** -10, 2.0 - 2.0 ** -23, 0.0, -2.0, -math.inf):
        for extra in (-1, 0, 1):
            s = torch.full((1, 2, 60 + 200), low)
            g = torch.Generator().manual_seed(extra + 5)
            for h in range(2):
                s[0, h, 60 + torch.randperm(200, generator=g)[:60 + extra]] = 2.0
            check_select(1, 2, 200, 64, 60, 0, BF, score=s)


def test_select_equal_and_special_scores():
    """Ties go to the lowest entry; zeros are one number, NaN is above infinity."""
    for pick in ([1.0], [0.0, -0.0], [math.inf, -math.inf, math.nan, 0.0, -0.0, -1.5, 1e-40, -1e-40, 3.0]):
        g = torch.Generator().manual_seed(len(pick))
        s = torch.tensor(pick)[torch.randint(0, len(pick), (2, 2, 40 + 90), generator=g)]
        check_select(2, 2, 90, 32, 40, 6, F32, score=s)
        check_select(2, 2, 90, 32, 40, 6, F32, score=s, pos=[20, 100], cached=True)


def check_step(B, H, Hkv, d, slots, recent, pos, dtype, seed=3, inplace=True, scale=None, score=None):
    bla = _bla()
    _say(f"evict step {B}x{H}/{Hkv}x{d} slots {slots} recent {recent} pos {pos} {dtype} in place {inplace}")
    q, k, v = normal(seed, B, H, d, dtype=dtype, std=1.5), normal(seed + 1, B, Hkv, d, dtype=dtype), normal(seed + 2, B, Hkv, d, dtype=dtype)
    ck, cv = normal(seed + 3, B, Hkv, slots, d, dtype=dtype), normal(seed + 4, B, Hkv, slots, d, dtype=dtype)
    score = weights(seed + 5, B, Hkv, slots) if score is None else score.clone()
    at = torch.full((B, Hkv, slots), -1)
    g = torch.Generator().manual_seed(seed + 6)
    for b in range(B):
        n = min(max(pos[b], 0), slots)
        ck[b, :, n:], cv[b, :, n:], score[b, :, n:] = math.nan, math.nan, math.nan
        for h in range(Hkv):  # a full cache holds the newest `recent` and some others
            step = max(1, (pos[b] - recent) // max(1, slots - recent))
            every = torch.arange(slots) * step if pos[b] >= slots else torch.arange(slots)
            if pos[b] >= slots:
                every[slots - recent:] = torch.arange(pos[b] - recent, pos[b])
                every = every[torch.randperm(slots, generator=g)]
            at[b, h, :n] = every[:n]
    gq, gk, gv, gck, gcv, gs, ga, gp = dev(q, k, v, ck, cv, score, at, torch.tensor(pos, dtype=torch.int64))
    more = {} if inplace else {"score_out": torch.full_like(gs, 9.0), "at_out": torch.full_like(ga, 9)}
    o, gs2, ga2 = bla.evict_step(gq, gk, gv, gck, gcv, gs, ga, recent, pos=gp, scale=scale, **more)
    torch.cuda.synchronize()
    assert (gs2 is gs) == inplace
    if not inplace:
        assert torch.equal(gs.cpu().nan_to_num(-7.0), score.nan_to_num(-7.0)) and torch.equal(ga.cpu(), at)
    o, os, oa, ok, ov = o.cpu(), gs2.cpu(), ga2.cpu(), gck.cpu(), gcv.cpu()
    u, sc = unit(dtype), 1 / math.sqrt(d) if scale is None else scale
    same = lambda x, y: torch.equal(x.nan_to_num(-7.0), y.nan_to_num(-7.0))  # noqa: E731
    for b in range(B):
        if pos[b] < 0:
            assert not o[b].any() and same(os[b], score[b]) and torch.equal(oa[b], at[b]) and same(ok[b], ck[b]) and same(ov[b], cv[b])
            continue
        rep, p = H // Hkv, pos[b]
        for h in range(Hkv):
            mine = p
            if p >= slots:
                may = [i for i in range(slots) if int(at[b, h, i]) < p - recent]
                mine = min(may, key=lambda i: (order_key(float(score[b, h, i])), i))
            n = min(p + 1, slots)
            rest = torch.tensor([i for i in range(n) if i != mine], dtype=torch.int64)
            for out, old, new in ((ok, ck, k), (ov, cv, v)):
                want = old[b, h].clone()
                want[mine] = new[b, h]
                assert same(out[b, h], want)
            want = at[b, h].clone()
            want[mine] = p
            assert torch.equal(oa[b, h], want)
            heads = slice(h * rep, (h + 1) * rep)
            ref = row(q[b, heads, None], k[b, h:h + 1, None], v[b, h:h + 1, None], 0, ENDLESS, 0, sc, front_k=ck[b, h:h + 1, rest], front_v=cv[b, h:h + 1, rest])
            close(o[b, heads, None], ref["o"], (u + ref["r"]) * ref["spread"] + u * ref["o"].abs(), f"o[{b}]")
            before = torch.cat([score[b, h, rest].to(F64), torch.zeros(1, dtype=F64)])[None]
            fine = torch.isfinite(before)
            got = torch.cat([os[b, h, rest], os[b, h, mine:mine + 1]])[None]
            close(got[fine][None], (before + ref["seen_by"])[fine][None], score_bound(ref, 1, rep, before.abs())[fine][None], f"score[{b}]")
            assert same(got[~fine], before.float()[~fine]) and same(os[b, h, n:], score[b, h, n:])


@pytest.mark.parametrize("inplace", [True, False])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("H,Hkv,d,slots,recent,pos", [
    (4, 4, 64, 44, 4, [0, 1, 43, 44, 45, 5000]),
    (8, 1, 32, 1, 0, [0, 1, 77]),                              # one slot: every token takes it
    (40, 2, 128, 130, 129, [0, 129, 130, 131, 1 << 40]),       # twenty heads to a key head; one slot that can go
    (4, 2, 64, 3000, 70, [2999, 3000, 3001, 100000]),          # parts of the cache
    (2, 2, 128, 300, 0, [-1, 5, 299, 300, -(1 << 62)]),        # rows without a token
    (4, 2, 64, 960, 30, [959, 960, 40, 90000]),                # the longest cache of one launch, and the next
    (4, 2, 64, 961, 30, [960, 961, 40, 90000]),
    (4, 2, 64, 480, 30, [479, 480, 40, 90000]),                # in float32
    (16, 2, 128, 1024, 30, [1023, 1024, 40, 90000] * 17),      # the most scores that stay on the chip, or more
    (32, 2, 128, 240, 30, [239, 240, 40, 90000]),
    (4, 2, 64, 2048, 30, [2047, 2048, 40, 90000] * 17),        # with more rows
    (4, 2, 64, 2049, 30, [2048, 2049, 40, 90000] * 17),
    (100, 1, 32, 2100, 10, [2500, -1, 7]),                     # more heads than the sums take at a time
])
def test_step(dtype, inplace, H, Hkv, d, slots, recent, pos):
    check_step(len(pos), H, Hkv, d, slots, recent, pos, dtype, inplace=inplace)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_step_many_rows(dtype):
    """Enough rows that a workgroup has a key head's slots and heads to itself."""
    check_step(300, 4, 2, 64, 200, 20, [(b * 37) % 450 - 1 for b in range(300)], dtype)
    check_step(300, 4, 2, 32, 70, 3, [(b * 37) % 450 - 1 for b in range(300)], dtype, inplace=False, scale=-0.3)


def test_step_equal_and_special_scores():
    for pick in ([1.0], [0.0, -0.0], [math.inf, math.nan, 0.0, -0.0, 3.0], [math.nan], [math.inf]):
        g = torch.Generator().manual_seed(len(pick))
        s = torch.tensor(pick)[torch.randint(0, len(pick), (4, 2, 50), generator=g)]
        check_step(4, 4, 2, 32, 50, 7, [50, 51, 70, 500], F32, score=s)


@pytest.mark.parametrize("dtype,heads,slots", [(BF, 8, 1000), (F32, 8, 1024), (F32, 9, 1000)])
def test_step_scores_in_lds(dtype, heads, slots):
    """Wide heads whose scores fill what LDS has for them, and one head more than that: 512 rows, of which a few have tokens."""
    bla = _bla()
    B, d = 512, 128
    _say(f"evict step 512x{heads}/1x128 slots {slots} {dtype}")
    g = torch.Generator(device="cuda").manual_seed(5)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g).to(dtype)  # noqa: E731
    q, k, v, ck, cv = rand(B, heads, d), rand(B, 1, d), rand(B, 1, d), rand(B, 1, slots, d), rand(B, 1, slots, d)
    score, at = torch.rand(B, 1, slots, device="cuda", generator=g), torch.arange(slots, device="cuda").expand(B, 1, slots).contiguous()
    pos = torch.full((B,), -1, dtype=torch.int64)
    some = {3: 10, 77: slots - 1, 300: slots, 511: slots + 5}
    for b, p in some.items():
        pos[b] = p
    before = [x.cpu() for x in (ck, cv, score)]
    o, score, at = bla.evict_step(q, k, v, ck, cv, score, at, 4, pos=pos.cuda())
    u = unit(dtype)
    for b, p in some.items():
        old_k, old_v, old = (x[b] for x in before)
        mine = p if p < slots else int(old[0, :min(slots, p - 4)].argmin())
        n = min(p + 1, slots)
        rest = torch.tensor([i for i in range(n) if i != mine])
        ref = row(q[b, :, None].cpu(), k[b, :, None].cpu(), v[b, :, None].cpu(), 0, ENDLESS, 0, 1 / math.sqrt(d), front_k=old_k[:, rest], front_v=old_v[:, rest])
        close(o[b, :, None].cpu(), ref["o"], (u + ref["r"]) * ref["spread"] + u * ref["o"].abs(), f"o[{b}]")
        was = torch.cat([old[0, rest].to(F64), torch.zeros(1, dtype=F64)])[None]
        got = torch.cat([score[b, 0, rest.cuda()], score[b, 0, mine:mine + 1]])[None].cpu()
        close(got, was + ref["seen_by"], score_bound(ref, 1, heads, was), f"score[{b}]")
        assert int(at[b, 0, mine]) == p
    assert not o[torch.tensor([b for b in range(B) if b not in some])].any()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_prompt_then_tokens(dtype):
    """A prompt, the tokens of it that stay, and single tokens: each token's score and the cache against a token-by-token recurrence in float64, whose choice
    of the slot that goes is taken from the kernel's scores (two scores may differ by less than their bound)."""
    bla = _bla()
    B, H, Hkv, d, slots, recent, L = 2, 4, 2, 32, 24, 6, 60
    q, k, v = (normal(80 + i, B, h, L, d, dtype=dtype, std=1.5 - 0.5 * (i > 0)) for i, h in enumerate((H, Hkv, Hkv)))
    gq, gk, gv = dev(q, k, v)
    n = 40
    first = [x[:, :, :n].contiguous() for x in (gq, gk, gv)]
    _, _, after = bla.evict_forward(*first, slots)
    ck, cv, score, at = bla.evict_select(first[1], first[2], after, slots, recent)
    u = unit(dtype)
    where, tally = at.cpu(), score.cpu().to(F64)
    for t in range(n, L):
        seen = score.cpu()
        o, score, at = bla.evict_step(*(x[:, :, t].contiguous() for x in (gq, gk, gv)), ck, cv, score, at, recent, t0=t)
        for b in range(B):
            for h in range(Hkv):
                may = [i for i in range(slots) if int(where[b, h, i]) < t - recent]
                mine = min(may, key=lambda i: (float(seen[b, h, i]), i))
                where[b, h, mine], tally[b, h, mine] = t, 0.0
                heads = slice(2 * h, 2 * h + 2)
                rest = torch.tensor([i for i in range(slots) if i != mine])
                ref = row(q[b, heads, t:t + 1], k[b, h:h + 1, t:t + 1], v[b, h:h + 1, t:t + 1], 0, ENDLESS, 0, 1 / math.sqrt(d),
                          front_k=k[b, h:h + 1, where[b, h, rest]], front_v=v[b, h:h + 1, where[b, h, rest]])
                close(o[b, heads, None].cpu(), ref["o"], (u + ref["r"]) * ref["spread"] + u * ref["o"].abs(), f"o[{b}] at {t}")
                tally[b, h, rest] += ref["seen_by"][0, :-1]
                tally[b, h, mine] += ref["seen_by"][0, -1]
        assert torch.equal(at.cpu(), where)
        # each step adds its own rounding of what is there: (r + 2^-23) a step, r below 2e-5 here
        close(score.cpu(), tally, (2e-5 + 2.0 ** -23) * (t - n + 2) * tally.abs(), f"scores at {t}")
