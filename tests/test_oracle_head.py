"""The oracle of vmoe_head_loss against differences and plain cases, on the CPU."""
import numpy as np
import pytest

from oracle import head


def _case(shared, seed=0):
    rng = np.random.default_rng(seed)
    T, N, V, d, K = 2, 4, 7, 3, 3
    z, w = rng.normal(size=(T, N, d)), rng.normal(size=(V, d) if shared else (T, V, d))
    label = rng.integers(0, V, size=(T, N))
    label[0, 1] = -1
    tidx = rng.integers(0, V, size=(T, N, K))
    tidx[1, 0] = [2, 5, 2]  # an index twice
    tidx[0, 2, 1] = V
    tidx[1, 3] = -1
    tlogit = rng.normal(size=(T, N, K))
    tlogit[0, 3, 2] = -np.inf
    return z, w, label, tidx, tlogit


@pytest.mark.parametrize("shared", [False, True])
def test_gradient_is_that_of_differences(shared):
    z, w, label, tidx, tlogit = _case(shared)
    rng = np.random.default_rng(1)
    T, N = label.shape
    dce, dlse, dkl = (rng.normal(size=(T, N)) for _ in range(3))
    tau = 1.7

    def total(z, w):
        r = head.loss(z, w, label, tidx, tlogit, tau)
        return (dce * r["ce"] + dlse * r["lse"] * r["has"] + dkl * r["kl"]).sum()
    r = head.loss(z, w, label, tidx, tlogit, tau)
    dl, size = head.dlogits(r, label, tidx, tau, dce, dlse, dkl)
    dz, dw = head.back(dl, z, w, r["has"] | r["taught"])
    assert np.all(np.abs(dl) <= size + 1e-12)
    h = 1e-6
    for a, g in ((z, dz), (w, dw)):
        for at in np.ndindex(a.shape):
            keep = a[at]
            a[at] = keep + h
            up = total(z, w)
            a[at] = keep - h
            dn = total(z, w)
            a[at] = keep
            assert abs((up - dn) / (2 * h) - g[at]) < 1e-7


def test_plain_cases():
    z, w, label, tidx, tlogit = _case(False, 3)
    r = head.loss(z, w, label)
    assert r["ce"][0, 1] == 0 and r["lse"][0, 1] == 0
    p = np.exp(r["logits"]) / np.exp(r["logits"]).sum(axis=2, keepdims=True)
    assert np.allclose(r["ce"][1], -np.log(np.take_along_axis(p[1], label[1][:, None], 1)[:, 0]))
    # a teacher that is the student: no divergence, no gradient
    full = np.broadcast_to(np.arange(7), (2, 4, 7))
    r = head.loss(z, w, None, full, np.einsum("tnd,tvd->tnv", z, w), 2.0)
    assert np.allclose(r["kl"], 0)
    dl, _ = head.dlogits(r, None, full, 2.0, dkl=np.ones((2, 4)))
    assert np.allclose(dl, 0)
