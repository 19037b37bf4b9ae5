"""The fp64 oracle of the balance losses, block norms and AdamW against central differences and
hand-made values (CPU)."""
import numpy as np
import pytest

from oracle import training as tr


def _diff(f, a, h=1e-5):
    """Central differences of the scalar f by every element of a."""
    g = np.zeros_like(a)
    for i in np.ndindex(*a.shape):
        keep = a[i]
        a[i] = keep + h
        hi = f()
        a[i] = keep - h
        lo = f()
        a[i] = keep
        g[i] = (hi - lo) / (2 * h)
    return g


@pytest.mark.parametrize("masked", [False, True])
def test_balance_gradient_by_differences(masked):
    r = np.random.RandomState(3)
    T, N, E, k = 2, 5, 4, 2
    x = r.randn(T, N, E)
    idx = np.argsort(-x, axis=2)[:, :, :k]  # held fixed
    mask = np.ones((T, N), np.uint8)
    if masked:
        mask[0, 2:] = 0
        mask[1] = 0
    dl = r.rand(T, 3)
    f = lambda: float((tr.balance(x, idx, mask)["loss"] * dl).sum())  # noqa: E731
    got, _, _ = tr.balance_bwd(tr.balance(x, idx, mask), dl)
    # third derivatives of O(1), h = 1e-5: 1e-10, and rounding 1e-16 / 1e-5
    assert np.max(np.abs(got - _diff(f, x))) < 1e-8
    if masked:
        assert np.all(got[1] == 0) and np.all(tr.balance(x, idx, mask)["loss"][1] == 0)


def test_balance_of_an_even_load_is_one():
    x = np.zeros((1, 8, 4))
    idx = np.stack([np.arange(8) % 4, (np.arange(8) + 1) % 4], axis=1)[None]
    f = tr.balance(x, idx)
    assert np.allclose(f["loss"][0], [1.0, 0.0, np.log(4) ** 2]) and f["count"].tolist() == [[4, 4, 4, 4]]


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("part", ["pre", "post", "both"])
def test_block_norm_gradient_by_differences(rms, post, part):
    r = np.random.RandomState(5)
    T, N, d, rho, eps = 2, 3, 8, 1.3, 1e-3
    x, y = r.randn(T, N, d), 2 * r.randn(T, N, d)
    pw, pb, gate, qw, qb = (r.randn(T, d) for _ in range(5))
    dz, du = r.randn(T, N, d), r.randn(T, N, d)
    if part == "pre":
        y = None

    def f():
        z = x if y is None else tr.block_z(x, y, pw if post else None, pb if post else None, gate, rho, rms, post, eps)
        s = float((dz * z).sum())
        return s if part == "post" else s + float((du * tr.norm(z, qw, qb, rms, eps)).sum())

    z = x if y is None else tr.block_z(x, y, pw if post else None, pb if post else None, gate, rho, rms, post, eps)
    got, _ = tr.block_bwd(y, z, pw if post else None, pb if post else None, gate, qw, dz, None if part == "post" else du, rho, rms,
                          post, eps)
    by = {"dx": x}
    if part != "post":
        by.update(dpre_w=qw, dpre_b=qb)
    if y is not None:
        by.update(dy=y, dgate=gate)
        if post:
            by.update(dpost_w=pw, dpost_b=pb)
    for n, a in by.items():
        assert np.max(np.abs(got[n] - _diff(f, a))) < 1e-6, n


def test_adamw_first_step_moves_by_the_rate():
    """m / (1 - b1) = g and v / (1 - b2) = g^2 after one step: the update is lr sign(g)."""
    g = np.array([3.0, -0.25, 1e-3])
    p, m, v, _ = tr.adamw(np.ones(3), g, np.zeros(3), np.zeros(3), 1, 0.1, 0.9, 0.999, 1e-12, weight_decay=0.5)
    assert np.allclose(p, 1 - 0.1 * 0.5 - 0.1 * np.sign(g)) and np.allclose(m, 0.1 * g) and np.allclose(v, 1e-3 * g * g)


def test_dither_is_even_and_independent():
    """Both halves of the hash: uniform, and uncorrelated with each other, the next element's, the next
    step's and the next tensor's.  2^16 draws: means within 4.5 sigma of 1/2, correlations within 4.5 / 2^8."""
    n = 1 << 16
    for seed, step in ((0, 1), (1, 1), (0, 2), (123, 1000)):
        lo, hi = (b / 65536.0 for b in tr.dither_bits(n, 0, step, seed))
        others = [hi, np.roll(lo, 1), tr.dither_bits(n, 0, step + 1, seed)[0], tr.dither_bits(n, 1, step, seed)[0]]
        for a in (lo, hi):
            assert abs(a.mean() + 0.5 / 65536 - 0.5) < 4.5 / np.sqrt(12 * n)
            assert abs(a.std() - 12 ** -0.5) < 0.005
        for o in others:
            assert abs(np.corrcoef(lo, o)[0, 1]) < 4.5 / 256


def test_e4m3_encoding_keeps_the_mean_and_exact_values():
    """Values that e4m3 has are kept; others go to a neighbour, the value in the mean."""
    exact = np.array([448.0, 1.0, -0.015625, 2.0 ** -9, 0.0, 240.0, -3.5])
    for bits in (0, 65535):
        q, scale, _, _ = tr.e4m3_encode(exact, np.full(exact.size, bits))
        assert scale[0] == 1.0 and np.array_equal(q, exact)
    for a in (1.05, 300.0, 0.01, 1e-3):
        v = np.full(65536, a)
        v[::256] = 448.0
        q, _, _, grid = tr.e4m3_encode(v, np.arange(65536))
        body = np.ones(65536, bool)
        body[::256] = False
        assert len(np.unique(q[body])) == 2 and abs(q[body].mean() - a) < grid[1] * 2.0 ** -7
