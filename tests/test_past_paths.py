"""The forms that a call over a ring, a prefix or a bounded cache may take, each at its borders: which form a shape takes is told from its workspace's size (on the
host), and its results are compared with the definition on the GPU."""
import ctypes
import math

import pytest
import torch

import paper_2606_09862_amd as bla
import test_gpu_bias as bias
import test_gpu_evict as evict
import test_gpu_prefix as prefix
from test_gpu_window import dev, normal

BF, F32 = torch.bfloat16, torch.float32
EDGES = bias.LOG + bias.FAR


def align(n):
    return (n + 255) // 256 * 256


def window_of(B, H, Hkv, d, window, sinks, dtype):
    return bla.WindowParams(B, H, Hkv, 1, d, window, sinks, int(dtype == BF), 0, 0.0)


def some(B, active, idle=-1):
    """B rows of which a few have tokens, spread over them."""
    pos = [idle] * B
    for i, p in enumerate(active):
        pos[(i * 31 + 5) % B] = p
    assert sum(p >= 0 for p in pos) == len(active)
    return pos


# One launch with a workgroup of eight waves to a key head, where the key heads alone need two parts to fill the device: 132 rows of two.
RINGS = [
    (132, 4, 2, 64, 2040, 8, BF, "one"), (132, 4, 2, 64, 2041, 8, BF, "parts"),
    (132, 4, 2, 64, 2040, 8, F32, "one"), (132, 4, 2, 64, 2041, 8, F32, "parts"),    # 2048 slots and 512 KiB
    (132, 4, 2, 128, 1020, 4, F32, "one"), (132, 4, 2, 128, 1021, 4, F32, "parts"),  # 512 KiB
    (128, 4, 2, 64, 1020, 5, BF, "parts"), (129, 4, 2, 64, 1020, 5, BF, "one"),      # from 257 key heads on
    (9, 40, 2, 64, 954, 6, BF, "one"),                                               # two groups of heads to a key head
]


@pytest.mark.parametrize("B,H,Hkv,d,window,sinks,dtype,form", RINGS)
def test_form_of_a_biased_step(B, H, Hkv, d, window, sinks, dtype, form):
    need = bla.lib().bla_bias_step_workspace_size(ctypes.byref(window_of(B, H, Hkv, d, window, sinks, dtype)))
    assert (need == 0) == (form == "one")


@pytest.mark.gpu
@pytest.mark.parametrize("B,H,Hkv,d,window,sinks,dtype,form", RINGS)
def test_biased_step(B, H, Hkv, d, window, sinks, dtype, form):
    slots = window + sinks
    bias.test_step(dtype, H, Hkv, d, window, sinks, some(B, [slots - 1, 40, slots, 90000, 0, slots + 31]), EDGES)


# The scores of a fused step in LDS or in the workspace, and parts.
CACHES = [
    (132, 4, 2, 64, 2048, 30, BF, "lds"), (132, 4, 2, 64, 2049, 30, BF, "parts"),
    (132, 4, 2, 64, 2048, 30, F32, "lds"), (132, 4, 2, 64, 2049, 30, F32, "parts"),
    (132, 16, 2, 128, 1024, 30, BF, "lds"), (132, 18, 2, 128, 1024, 30, BF, "memory"),   # 32 KiB of scores
    (132, 8, 2, 128, 1024, 30, F32, "lds"), (132, 10, 2, 128, 1024, 30, F32, "memory"),  # 16 KiB
    (6, 32, 2, 64, 960, 30, BF, "memory"), (6, 32, 2, 32, 960, 30, F32, "memory"),
    (6, 40, 2, 64, 960, 30, BF, "parts"),                                                # two groups of heads: the sums need a second launch
]


@pytest.mark.parametrize("B,H,Hkv,d,slots,recent,dtype,form", CACHES)
def test_form_of_an_evicting_step(B, H, Hkv, d, slots, recent, dtype, form):
    p = bla.EvictParams(B, H, Hkv, 1, d, slots, recent, int(dtype == BF), 0, 0.0)
    need = bla.lib().bla_evict_step_workspace_size(ctypes.byref(p))
    slot, scores = align(B * Hkv * 4), align(B * H * ((slots + 31) // 32 * 32) * 4)
    assert (need == slot) == (form == "lds") and (need == slot + scores) == (form == "memory") and (need > slot + scores) == (form == "parts")


@pytest.mark.gpu
@pytest.mark.parametrize("B,H,Hkv,d,slots,recent,dtype,form", CACHES)
def test_evicting_step(B, H, Hkv, d, slots, recent, dtype, form):
    pos = some(B, [slots - 1, slots, 40, 90000, 0, slots + 31][:min(6, B)])
    evict.check_step(B, H, Hkv, d, slots, recent, pos, dtype)


# A step behind a prefix: in one launch, the prefix's queries as a ring's heads, or in tiles.
PREFIXES = [
    (1, 1, 24, 1, 64, 448, 500, 12, [900], None, BF, "one"),         # two groups of heads, the most tokens
    (2, 2, 24, 1, 32, 448, 500, 12, [900, 3], [448, 33], F32, "one"),
    (2, 1, 2, 1, 64, 448, 500, 12, [3, 900], None, BF, "one"), (2, 1, 2, 1, 64, 449, 500, 12, [3, 900], None, BF, "few"),
    (2, 1, 2, 1, 32, 448, 500, 12, [3, 900], None, F32, "one"), (2, 1, 2, 1, 32, 449, 500, 12, [3, 900], None, F32, "few"),
    (6, 2, 8, 1, 64, 3000, 40, 4, [3, 900, -1, 0, 43, 44], [3000, 1777], BF, "few"),     # 24 queries: the second block has eight
    (6, 2, 16, 2, 128, 2000, 40, 4, [3, -1, 900, 0, 43, 44], [1, 2000], F32, "few"),
    (12, 2, 10, 2, 64, 1500, 40, 4, [3, 900, 7, 0, -1, 44], [1500, 0], BF, "few"),       # 30: a block begins inside a row
    (8, 2, 8, 1, 32, 2500, 40, 4, [3, 900, -1, 0], [2500, 64], BF, "few"),               # 32, the most
    (11, 1, 3, 1, 64, 2500, 40, 4, [3, 900, -1, 0], None, BF, "tiles"),                  # 33
]


@pytest.mark.parametrize("B,G,H,Hkv,d,P,window,sinks,pos,plen,dtype,form", PREFIXES)
def test_form_of_a_step_behind_a_prefix(B, G, H, Hkv, d, P, window, sinks, pos, plen, dtype, form):
    p = bla.PrefixParams(window_of(B, H, Hkv, d, window, sinks, dtype), P, G)
    need = bla.lib().bla_prefix_step_workspace_size(ctypes.byref(p))
    queries = B // G * (H // Hkv)
    assert (need == 0) == (form == "one") and (form == "tiles") == (queries > 32)


@pytest.mark.gpu
@pytest.mark.parametrize("B,G,H,Hkv,d,P,window,sinks,pos,plen,dtype,form", PREFIXES)
def test_step_behind_a_prefix(B, G, H, Hkv, d, P, window, sinks, pos, plen, dtype, form):
    prefix.check_step(B, G, H, Hkv, d, P, window, sinks, pos, dtype, plen)


def growing(G, Hkv, P, d, dtype, plen, seed):
    """Prefixes whose keys grow along them, so that a query's largest score moves from tile to tile, no two tiles alike."""
    g = torch.linspace(0.1, 3.0, max(P, 1))[:P, None]
    pk, pv = (normal(seed, G, Hkv, P, d, dtype=F32) * g).to(dtype), normal(seed + 1, G, Hkv, P, d, dtype=dtype)
    n = [P if plen is None else min(max(plen[x], 0), P) for x in range(G)]
    for x in range(G):
        pk[x, :, n[x]:], pv[x, :, n[x]:] = math.nan, math.nan
    return pk, pv, n


# (rows, prefixes, heads, key heads, tokens, tiles of 64 to a part): the tiles of a part pass through two buffers, with one or two groups of waves
WALKS = [(48, 16, 48, 4, 1111, 5), (64, 64, 132, 4, 700, 11), (20, 2, 16, 2, 9000, 3), (5, 5, 70, 2, 3333, 3)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (BF, 32), (F32, 64), (F32, 128), (F32, 32)])
@pytest.mark.parametrize("B,G,H,Hkv,P,tiles", WALKS)
def test_a_prefix_of_several_tiles_to_a_part(monkeypatch, dtype, d, B, G, H, Hkv, P, tiles):
    need = bla.lib().bla_prefix_step_workspace_size(ctypes.byref(bla.PrefixParams(window_of(B, H, Hkv, d, 30, 2, dtype), P, G)))
    parts = need // (B * H * (d + 2) * 4) - 1                  # one is the ring's
    assert parts <= -(-P // 64) // 2 and -(-(-(-P // 64)) // parts) == tiles
    monkeypatch.setattr(prefix, "prefixes", growing)
    plen = [P - 37 * g % P if g else P for g in range(G)]
    prefix.check_step(B, G, H, Hkv, d, P, 30, 2, some(B, [40, 3, 31, 1000, 0]), dtype, plen)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d", [(BF, 64), (F32, 64), (BF, 128)])
def test_biased_backward_of_many_blocks(dtype, d):
    """More blocks of queries and keys than two workgroups to a compute unit, whose order is turned for every second 256 of them: all gradients, padded rows and sinks, and
    a workspace that held NaN."""
    B, H, L, window, sinks = 9, 16, 520, 300, 4
    lengths = [520, 1, 333, 0, 520, 519, 64, 520, 200]
    per = -(-L // (128 if d < 128 else 64))
    assert B * H * per > 512 and B * H * per % 256
    bias.check_backward(B, H, H, L, d, window, sinks, dtype, bias.LOG, lengths=lengths)
    q, k, v, dO = (normal(70 + i, B, H, L, d, dtype=dtype).cuda() for i in range(4))
    b, n = normal(80, H, len(bias.LOG) + 1, dtype=F32).cuda(), dev(torch.tensor(lengths, dtype=torch.int32))[0]
    o, lse, _, _ = bla.bias_forward(q, k, v, b, bias.LOG, window, sinks, lengths=n, want_lse=True)
    p = bla.WindowParams(B, H, H, L, d, window, sinks, int(dtype == BF), 0, 0.0)
    need = bla.lib().bla_bias_backward_workspace_size(ctypes.byref(p), len(bias.LOG) + 1)
    args = (q, k, v, o, lse, dO, b, bias.LOG, window, sinks)
    want = bla.bias_backward(*args, lengths=n, workspace=torch.zeros(need // 4, device="cuda").view(torch.uint8))
    got = bla.bias_backward(*args, lengths=n, workspace=torch.full((need // 4,), math.nan, device="cuda").view(torch.uint8))
    assert all(torch.isfinite(x).all() and torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.gpu
@pytest.mark.parametrize("slots", [300, 3000])  # one launch, and parts
def test_evicting_step_with_one_result_in_place(slots):
    """Scores in place and positions elsewhere, and the other way round: the same results, and what is not in place stays as it was."""
    B, H, Hkv, d = 4, 4, 2, 64
    pos = torch.tensor([slots + 9, 5, -1, slots], device="cuda")
    x = [normal(90 + i, *s).cuda() for i, s in enumerate(((B, H, d), (B, Hkv, d), (B, Hkv, d), (B, Hkv, slots, d), (B, Hkv, slots, d)))]
    score, at = evict.weights(96, B, Hkv, slots).cuda(), torch.arange(slots, device="cuda").expand(B, Hkv, slots).contiguous()

    def step(**more):
        s, a = score.clone(), at.clone()
        got = bla.evict_step(*x[:3], x[3].clone(), x[4].clone(), s, a, 7, pos=pos, **more)
        return s, a, got

    _, _, want = step()
    s, a, got = step(at_out=torch.full_like(at, 9))
    assert got[1] is s and torch.equal(a, at) and all(torch.equal(y, z) for y, z in zip(got, want))
    s, a, got = step(score_out=torch.full_like(score, 9.0))
    assert got[2] is a and torch.equal(s, score) and all(torch.equal(y, z) for y, z in zip(got, want))
