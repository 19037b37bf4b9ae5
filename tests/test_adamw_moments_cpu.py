"""AdamW with 8-bit moments over many steps, on the oracle (CPU): what its definition does to the updates.

The bound.  Roundings are unbiased where a value is above one step, so moments m' and roots r' as they are read
back scatter around the exact m and r.  The stored root forgets over 1 / (1 - b2) = 1000 steps: n steps of e4m3
below its normal range move to a neighbour with probability n (1 - b2) / 2 a step, a variance of n / 2 in the
long run, so n = 4 may be found at 1 (two deviations) and n = 8 at 2 (three): r' >= r / 4, and never 0.  The
moment forgets over 10 steps: roundings of variance S^2 / 4, S = 2^-9 of its scale, add up to S^2 / 4 / (1 -
b1^2), 1.15 S, three deviations 3.4 S.  So m' / r' <= 4 (9/8 |m| / r) + 3.4 S_m / S_v, and S_m / S_v, the block's
largest |m| over its largest r, is at most the largest |m| / r: 8 times that of exact moments in all.
The paths: 1 / r' is in the mean at most twice 1 / r (n = 1 or 2), the moment's scatter is at most of the size
of its own update, the same random walk: sqrt(2^2 + 1) < 3 times the exact path's.
"""
import numpy as np
import pytest

from oracle import training as tr

B1, B2, EPS = 0.9, 0.999, 1e-8


def _run(grads, eight, seed=3):
    """(largest |update| / lr of each step, sum of the updates / lr) for gradients [steps, n]."""
    n = grads.shape[1]
    p, m, v, largest = np.zeros(n), np.zeros(n), np.zeros(n), []
    for t, g in enumerate(grads, 1):
        p, m, v, upd = tr.adamw(p, g, m, v, t, 1.0, B1, B2, EPS)
        largest.append(upd.max())
        if eight:
            lo, hi = tr.dither_bits(n, 0, t, seed)
            q, s, _, _ = tr.e4m3_encode(m, lo)
            m = q * np.repeat(s, 256)[:n]
            q, s, _, _ = tr.e4m3_encode(np.sqrt(v), hi, root=True)
            v = (q * np.repeat(s, 256)[:n]) ** 2
    return np.array(largest), p


def _spread(top, ratio, steps=400, n=64 * 256):
    """Element scales spread evenly in the logarithm over `ratio` within each block, `top` the largest."""
    r = np.random.RandomState(1)
    scale = top * ratio ** -r.rand(n)
    return scale * r.randn(steps, n)


def _sparse(low, steps=600, n=16 * 256):
    """One element of a block at 1, the others at `low`, where three steps of ten have a gradient."""
    r = np.random.RandomState(2)
    g = low * r.randn(steps, n) * (r.rand(steps, n) < 0.3)
    g[:, ::256] = r.randn(steps, n // 256)
    return g


@pytest.mark.parametrize("grads", [lambda: _spread(0.01, 1e6), lambda: _spread(0.1, 1e6), lambda: _spread(1.0, 1e5),
                                   lambda: _spread(1.0, 1e6), lambda: _sparse(2.0 ** -14), lambda: _sparse(2.0 ** -16)],
                         ids=["spread_1e-2_1e6", "spread_1e-1_1e6", "spread_1_1e5", "spread_1_1e6", "sparse_2^-14", "sparse_2^-16"])
def test_updates_stay_near_those_of_exact_moments(grads):
    g = grads()
    exact, pe = _run(g, False)
    eight, p8 = _run(g, True)
    assert eight.max() <= 8 * exact.max(), (eight.max(), exact.max())
    assert np.sqrt((p8 ** 2).mean()) <= 3 * np.sqrt((pe ** 2).mean())


def test_a_positive_root_keeps_a_step_and_zero_stays_zero():
    v = np.array([448.0, 2.0 ** -9, 2.0 ** -10, 2.0 ** -30, 0.0, 1.5 * 2.0 ** -9])
    for bits in (0, 65535):
        q, scale, _, _ = tr.e4m3_encode(v, np.full(v.size, bits), root=True)
        assert scale[0] == 1.0 and q[0] == 448.0 and q[4] == 0.0
        assert np.all(q[1:4] == 2.0 ** -9) and q[5] in (2.0 ** -9, 2.0 ** -8)
    q, scale, _, _ = tr.e4m3_encode(np.full(256, 2.0 ** -101), np.zeros(256, np.int64), root=True)
    assert scale[0] == 0 and np.all(q == 0)  # a block below the least scale
