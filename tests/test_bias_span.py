"""The distances between 32 keys and a wave's queries, which decide where the kernels of the learned bias take their biases from (csrc/bla_bias.h), against
the distances of all pairs; and every place of the table of near distances that may be read is one that is written."""
import itertools

import numpy as np

from host_probe import run

NEAR = 1024


def spans():
    """(first query, queries, first key, how much further the keys at negative indices are)."""
    for far, queries in itertools.product((0, 1, 30, 63, 64, 97, 173, 400, 900, 960, 1023, 5000), (16, 32)):
        for i0 in (*range(-160, 33), 96, 500, 1000, 1500):
            for qi in (0, 1, 15, 16, 47, 63, 64, 100, 127, 300, 1000, 1100):
                if qi + queries > i0:  # some query is at the keys or past them
                    yield qi, queries, i0, far


def test_spans_and_table():
    cases = list(spans())
    lasts = (0, 1, 2, 63, 64, 65, 113, 128, 300, 900, 959, 960, 961, 1023, 1024, 1 << 29)
    got = np.array([list(map(int, line.split())) for line in run("bias", [" ".join(map(str, c)) for c in cases])])
    ends = dict(zip(lasts, (int(line) for line in run("bias_table", map(str, lasts)))))
    assert len(got) == len(cases)
    several = 0
    for (qi, queries, i0, far), (lo, hi, near) in zip(cases, got):
        keys = np.arange(i0, i0 + 32)
        n = qi + np.arange(queries)[:, None] - keys[None] + np.where(keys < 0, far, 0)[None]
        assert hi >= n.max() and lo <= n.min(), (qi, queries, i0, far)
        if near:  # one run of distances: the ends are those of the pairs
            assert (keys >= 0).all() or (keys < 0).all()
            assert hi == n.max() and lo == n.min() and hi < NEAR and hi - lo < 63, (qi, queries, i0, far)
            for last in lasts:
                if lo < last <= hi:  # the ends may have different buckets
                    written = -(-ends[last] // 64) * 64
                    assert n.max() < written <= NEAR and n.min() >= -64, (qi, queries, i0, far, last)
                    several += 1
    assert several > 1000
