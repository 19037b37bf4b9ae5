"""The oracle of vmoe_gate against brute force and differences, on the CPU."""
import itertools

import numpy as np
import pytest

from oracle import gating


def test_choice_is_the_best_set_of_open_experts():
    """Every set of two experts in two of three groups: the chosen one has the largest sum of s + b."""
    rng = np.random.default_rng(0)
    x, b = rng.normal(size=(2, 5, 6)), 0.2 * rng.normal(size=(2, 6))
    ref = gating.choose(x, b, None, 2, 100, "sigmoid", 3, 2, 2)
    for t, n in itertools.product(range(2), range(5)):
        c = 1 / (1 + np.exp(-x[t, n])) + b[t]
        pair = max(itertools.combinations(range(3), 2), key=lambda g: sum(c[2 * i:2 * i + 2].sum() for i in g))
        may = [e for e in range(6) if e // 2 in pair]
        best = max(itertools.combinations(may, 2), key=lambda p: c[list(p)].sum())
        assert set(ref["idx"][t, n]) == set(best)
        assert abs(ref["gate"][t, n].sum() - 1) < 1e-12


def test_masked_tokens_and_switched_off_experts_take_no_place():
    x = np.zeros((1, 4, 3))
    x[0, :, 0] = -np.inf
    x[0, 2] = np.nan
    mask = np.array([[1, 0, 1, 1]])
    ref = gating.choose(x, None, mask, 3, 1, "softmax")
    assert ref["idx"][0].tolist() == [[1, 2, -1], [-1, -1, -1], [-1, -1, -1], [1, 2, -1]]
    assert ref["slot"][0].tolist() == [[0, 0, -1], [-1, -1, -1], [-1, -1, -1], [-1, -1, -1]]
    assert ref["demand"][0].tolist() == [0, 2, 2] and ref["load"][0].tolist() == [0, 1, 1]


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("renorm", [True, False])
def test_gradient_is_that_of_differences(score, renorm):
    rng = np.random.default_rng(3)
    T, N, E, d, k, scale = 2, 3, 6, 4, 2, 1.7
    x, w = rng.normal(size=(T, N, d)), rng.normal(size=(T, d, E))
    dy, ye = rng.normal(size=(T, N, d)), rng.normal(size=(T, E, N, d))
    logits = np.einsum("tnd,tde->tne", x, w)
    bias = 0.1 * rng.normal(size=(T, E))
    ref = gating.choose(logits, bias, None, k, 1, score, 2, 1, 2, renorm, scale)

    def y_dot(l):
        s, _ = gating.scores(l, score)
        mine = np.take_along_axis(s, ref["idx"], axis=2)
        gate = scale * (mine / mine.sum(axis=2, keepdims=True) if renorm else mine)
        out = 0.0
        for t, n, j in itertools.product(range(T), range(N), range(k)):
            if ref["slot"][t, n, j] >= 0:
                out += gate[t, n, j] * (dy[t, n] * ye[t, ref["idx"][t, n, j], ref["slot"][t, n, j]]).sum()
        return out
    g = gating.choose_bwd(ref, logits, x, w, dy, ye, score, renorm, scale)
    h = 1e-6
    for at in itertools.product(range(T), range(N), range(E)):
        up, dn = logits.copy(), logits.copy()
        up[at] += h
        dn[at] -= h
        assert abs((y_dot(up) - y_dot(dn)) / (2 * h) - g["dlogits"][at]) < 1e-7
