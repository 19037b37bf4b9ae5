"""vmoe_balance and its gradient where the first expert lies far below the others, on a GB300.

Tolerances.  exp(x - max) is 2^((x - max) log2 e): a difference, the constant and a product, each within 2^-24 of
the exponent, so 2.5 x 2^-24 |x - max| of the value (1.5e-7), and ex2.approx adds 2^-22 of it.  The sum s is 1
to E, its terms weighted by their size: |x - max| p is at most 1 / e, so with the roundings of the adding
s is within 5e-7, and so is its reciprocal.  p: within 1e-6 + 1.5e-7 |x - max|, relative.
lse = max + log(s): log2 is within 2^-22 of itself (from s = 2 on; 2^-22 below), log2(E) at most, s within 5e-7, one
rounding: 5e-7 + (1 + log2 E) 1.7e-7 + 2^-24 |lse|, absolute - whatever lse itself is, 0 included.
"""
import numpy as np
import pytest
import torch

import paper_2608_16188_gb300 as vm
from gpu_helpers import np64
from oracle import training as tr

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__
    __graft_entry__.build()


def _inputs(T, N, E, k, gap, centre):
    """Logits whose first expert lies `gap` below the largest; with `centre` shifted so that lse is near 0.01."""
    g = torch.Generator().manual_seed(E + N + int(min(gap, 999)))
    x = 0.7 * torch.randn(T, N, E, generator=g)
    x[..., 0] = x[..., 1:].amax(dim=2) - gap
    if centre:
        x = (x.double() - torch.logsumexp(x.double(), dim=2, keepdim=True) + 0.01).float()
    return x, x.topk(k, dim=2).indices.to(torch.int32)


def _run(x, idx, dloss):
    T, N, E = x.shape
    p = vm.problem(T, N, 8, 8, E, idx.shape[2], 1.0, "f32")
    bad = lambda *s, dt=torch.float32: torch.full(s, -7, dtype=dt, device="cuda")  # noqa: E731
    o = dict(count=bad(T, E, dt=torch.int32), tokens=bad(T, dt=torch.int32), excess=bad(T, E), loss=bad(T, 3), dlogits=bad(T, N, E))
    ws = torch.empty(vm.vmoe_balance_workspace_size(p), dtype=torch.uint8, device="cuda")
    x = x.cuda()
    vm.vmoe_balance(p, x, idx.cuda(), None, o["count"], o["tokens"], o["excess"], o["loss"], ws)
    vm.vmoe_balance_bwd(p, x, None, o["count"], o["tokens"], o["excess"], dloss.cuda(), o["dlogits"])
    return o


@pytest.mark.parametrize("gap", [0.0, 20.0, 30.0, 40.0, 60.0, 68.0, 70.0, 100.0, float("inf")])
@pytest.mark.parametrize("E", [2, 5, 32, 256])
@pytest.mark.parametrize("centre", [False, True])
def test_a_first_expert_far_below_the_others(E, gap, centre):
    T, N, k = 2, 130, min(2, E - 1)
    x, idx = _inputs(T, N, E, k, gap, centre)
    for dloss in (torch.tensor([[0.0, 0.0, 1.0]] * T), torch.tensor([[0.5, 0.0, 0.0]] * T)):
        o = _run(x, idx, dloss)
        ref = tr.balance(x, idx)
        assert np.array_equal(o["count"].cpu().numpy(), ref["count"]) and int(o["tokens"][0]) == N
        top = np64(x).max(axis=2, keepdims=True)
        far = np.where(np.isneginf(np64(x)), 0.0, top - np64(x))
        rel = 1e-6 + 1.5e-7 * far
        off = 5e-7 + (1 + np.log2(E)) * 1.7e-7 + 2.0 ** -24 * np.abs(ref["lse"])
        # the z-loss: a mean of squares, its own sum and division within 1e-6
        tol = (2 * np.abs(ref["lse"]) * off + off * off).mean(axis=1) + 1e-6 * ref["loss"][:, 2]
        assert np.all(np.abs(np64(o["loss"][:, 2]) - ref["loss"][:, 2]) <= tol)
        d, c, z = tr.balance_bwd(ref, dloss)
        p = ref["prob"]
        # p (c - sum p c + z): p's error, the sum's (the mean of those of its terms), and a rounding each of
        # c less its mean and of the difference; z off by as much as lse
        spread = np.abs(c - c.mean(axis=2, keepdims=True)).max(axis=2, keepdims=True)
        tol = p * (rel * (2 * spread + np.abs(z)) + 2e-6 * spread + np64(dloss)[:, 2, None, None] * 2 / N * off[:, :, None]) + 1e-37
        err = np.abs(np64(o["dlogits"]) - d)
        assert np.all(err <= tol), float((err / tol).max())
