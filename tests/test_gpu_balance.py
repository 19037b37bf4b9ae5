"""vmoe_balance and vmoe_balance_bwd against the fp64 oracle, on a GB300.

Tolerances.  exp(x - max) is 2^((x - max) log2 e): the product's rounding is off by half a step of the
exponent, |x - max| log2(e) 2^-24 ln 2 relative, which with |x - max| <= 24 is 1.5e-6, and ex2.approx adds
2^-22; the row's sum and its reciprocal add a few 2^-24.  So p is within 2e-6, relative, of the oracle's, and
  dlogits = p (c - sum p c + z): within 2e-6 p (2 max|c| + |z|) of p's error, as much again for the sum's and
  for the roundings of c, z and the difference: 4e-6 p (2 max|c| + |z|) in all;
  excess: 2e-6 of the importance, and the fp32 sums' roundings: 4e-6 (importance + M / E);
  loss: sums of such values: 1e-5, relative (loss 1: with the excess' error, twice its square root).
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


def _problem(T, N, E, k):
    return vm.problem(T, N, 8, 8, E, k, 1.0, "f32")


def _inputs(T, N, E, k, seed=0, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    x = scale * torch.randn(T, N, E, generator=g)
    idx = x.topk(k, dim=2).indices.to(torch.int32)
    return x, idx, torch.rand(T, 3, generator=g) * torch.tensor([0.1, 0.1, 0.01])


def _outputs(T, N, E, fill=float("nan")):
    f32 = lambda *s: torch.full(s, fill, device="cuda")  # noqa: E731
    i32 = lambda *s: torch.full(s, -7, dtype=torch.int32, device="cuda")  # noqa: E731
    return dict(count=i32(T, E), tokens=i32(T), excess=f32(T, E), loss=f32(T, 3), dlogits=f32(T, N, E))


def _run(p, x, idx, mask, dloss, stream=None):
    o = _outputs(p.T, p.N, p.E)
    ws = torch.full((vm.vmoe_balance_workspace_size(p),), 255, dtype=torch.uint8, device="cuda")
    vm.vmoe_balance(p, x, idx, mask, o["count"], o["tokens"], o["excess"], o["loss"], ws, stream=stream)
    vm.vmoe_balance_bwd(p, x, mask, o["count"], o["tokens"], o["excess"], dloss, o["dlogits"], stream=stream)
    return o


def _check(o, x, idx, mask, dloss):
    ref = tr.balance(x, idx, mask)
    assert np.array_equal(o["count"].cpu().numpy(), ref["count"])
    assert np.array_equal(o["tokens"].cpu().numpy(), ref["tokens"])
    imp = ref["prob"].sum(axis=1)
    even = ref["tokens"][:, None] / x.shape[2]
    ex_tol = 4e-6 * (imp + even)
    assert np.all(np.abs(np64(o["excess"]) - ref["excess"]) <= ex_tol)
    m = np.maximum(ref["tokens"], 1)
    tol = 1e-5 * np.abs(ref["loss"])
    E = x.shape[2]
    tol[:, 1] += E / (m * m) * (2 * np.abs(ref["excess"]) * ex_tol + ex_tol ** 2).sum(axis=1)
    assert np.all(np.abs(np64(o["loss"]) - ref["loss"]) <= tol)
    d, c, z = tr.balance_bwd(ref, dloss)
    # the backward has the GPU's excess
    cc = np.abs(c).max(axis=2, keepdims=True) + (np.abs(np64(dloss)[:, 1]) * 2 * E / (m * m) * ex_tol.max(axis=1))[:, None, None] / 2e-6
    bound = 4e-6 * ref["prob"] * (2 * cc + np.abs(z)) + 1e-37
    assert np.all(np.abs(np64(o["dlogits"]) - d) <= bound)
    assert np.all(o["dlogits"].cpu().numpy()[~ref["on"]] == 0)
    return ref


# every width of a row (1 to 256 experts, whole and ragged vectors of four), lengths from one token on,
# slices that end inside a step of rows, top-1 to top-8
SHAPES = [(1, 1, 1, 1), (1, 1, 2, 2), (2, 3, 3, 1), (1, 197, 8, 2), (3, 130, 4, 2), (2, 65, 5, 3), (2, 33, 16, 2),
          (2, 300, 13, 2), (4, 1576, 32, 2), (2, 257, 31, 2), (3, 100, 64, 1), (1, 515, 60, 8), (2, 70, 128, 4),
          (2, 61, 97, 3), (4, 129, 256, 8), (3, 40, 255, 8), (1, 7001, 130, 2), (1024, 2, 1, 1), (17, 20, 60, 2)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_balance_parity(shape):
    T, N, E, k = shape
    x, idx, dloss = _inputs(T, N, E, k, seed=sum(shape))
    o = _run(_problem(*shape), x.cuda(), idx.cuda(), None, dloss.cuda())
    _check(o, x, idx, None, dloss)


@pytest.mark.parametrize("shape", [(4, 197, 8, 2), (3, 70, 60, 1), (3, 300, 256, 8), (3, 33, 6, 2)], ids=str)
def test_padding_and_switched_off_experts(shape):
    """Padding holds NaN and indices of -1; a task without tokens; an expert at -inf; tokens all at -inf."""
    T, N, E, k = shape
    x, idx, dloss = _inputs(T, N, E, k, seed=7)
    mask = torch.ones(T, N, dtype=torch.uint8)
    mask[0, N // 3:] = 0
    mask[1] = 0
    x[2, :, E // 2] = float("-inf")
    x[0, 1] = float("-inf")
    x[2, N - 1] = float("-inf")
    mask[2, 0] = 200  # any value but 0
    x[mask == 0] = float("nan")
    idx[mask == 0] = -1
    o = _run(_problem(*shape), x.cuda(), idx.cuda(), mask.cuda(), dloss.cuda())
    ref = _check(o, x, idx, mask, dloss)
    assert ref["tokens"][1] == 0 and torch.all(o["loss"][1] == 0) and torch.all(o["excess"][1] == 0)
    assert np.all(o["dlogits"].cpu().numpy()[2, :, E // 2] == 0)


def test_wide_and_huge_logits():
    """Logits of +-20 (the bound above), the type's lowest value, and values near its largest."""
    T, N, E, k = 2, 96, 12, 2
    x, idx, dloss = _inputs(T, N, E, k, seed=9)
    x = x.clamp(-3, 3) * 4.0
    x[0, :, 3] = torch.finfo(torch.float32).min
    x[1, 5] = 3e38
    x[1, 6] = -3e38
    dloss[:, 2] = 0.0
    o = _run(_problem(T, N, E, k), x.cuda(), idx.cuda(), None, dloss.cuda())
    ref = tr.balance(x, idx)
    # the squares of 3e38 overflow, in task 1 alone
    assert torch.isinf(o["loss"][1, 2]) and torch.isfinite(o["loss"][0]).all()
    o["loss"][1, 2], ref["loss"][1, 2] = 0.0, 0.0
    d, _, _ = tr.balance_bwd(ref, dloss)
    assert np.max(np.abs(np64(o["dlogits"]) - d)) <= 1e-5 * np.max(np.abs(d))
    assert np.array_equal(o["count"].cpu().numpy(), ref["count"])


def test_nan_stays_in_its_task():
    T, N, E, k = 3, 50, 8, 2
    x, idx, dloss = _inputs(T, N, E, k, seed=11)
    x[1, 7, 2] = float("nan")
    o = _run(_problem(T, N, E, k), x.cuda(), idx.cuda(), None, dloss.cuda())
    assert torch.isnan(o["loss"][1]).any() and torch.isnan(o["dlogits"][1, 7]).all()
    good = [0, 2]
    _check({n: v[good] for n, v in o.items()}, x[good], idx[good], None, dloss[good])


def test_indices_out_of_range_and_repeated_are_safe():
    T, N, E, k = 1, 40, 8, 2
    x, idx, dloss = _inputs(T, N, E, k, seed=13)
    idx[0, 0] = torch.tensor([8, -2147483648], dtype=torch.int32)
    idx[0, 1] = torch.tensor([2147483647, 3], dtype=torch.int32)
    idx[0, 2] = torch.tensor([5, 5], dtype=torch.int32)
    o = _run(_problem(T, N, E, k), x.cuda(), idx.cuda(), None, dloss.cuda())
    _check(o, x, idx, None, dloss)


def test_in_place_gradient_streams_graphs_and_determinism():
    T, N, E, k = 5, 400, 32, 2
    p = _problem(T, N, E, k)
    x, idx, dloss = (v.cuda() for v in _inputs(T, N, E, k, seed=15))
    a = _run(p, x, idx, None, dloss)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b = _run(p, x, idx, None, dloss, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a[n], b[n]) for n in a)
    y = x.clone()  # dlogits over the logits
    vm.vmoe_balance_bwd(p, y, None, a["count"], a["tokens"], a["excess"], dloss, y)
    assert torch.equal(y, a["dlogits"])
    o = _outputs(T, N, E)
    ws = torch.empty(vm.vmoe_balance_workspace_size(p), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vm.vmoe_balance(p, x, idx, None, o["count"], o["tokens"], o["excess"], o["loss"], ws)
        vm.vmoe_balance_bwd(p, x, None, o["count"], o["tokens"], o["excess"], dloss, o["dlogits"])
    for scale in (1.0, -0.5):
        x.mul_(scale)
        graph.replay()
        torch.cuda.synchronize()
        c = _run(p, x, idx, None, dloss)
        torch.cuda.synchronize()
        assert all(torch.equal(o[n], c[n]) for n in o)


def test_losses_against_differences():
    """The kernels' gradient against central differences of the kernels' own losses.  h = 0.02 on losses of
    O(1) / N: fp32 losses within 1e-6 give differences within 1e-6 / 0.02 = 5e-5; the curvature's term is
    h^2 / 6 times a third derivative below the gradient's own scale."""
    T, N, E, k = 1, 4, 6, 2
    p = _problem(T, N, E, k)
    x, idx, dloss = _inputs(T, N, E, k, seed=17)
    dloss = torch.tensor([[0.5, 0.5, 0.1]])
    idx, dl = idx.cuda(), dloss.cuda()
    grad = np64(_run(p, x.cuda(), idx, None, dl)["dlogits"])
    for n in range(N):
        for e in range(E):
            v = []
            for h in (0.02, -0.02):
                y = x.clone()
                y[0, n, e] += h
                v.append(float((_run(p, y.cuda(), idx, None, dl)["loss"].double() * dl.double()).sum()))
            assert abs((v[0] - v[1]) / 0.04 - grad[0, n, e]) < 2e-4


@pytest.mark.parametrize("E", [7, 32, 256])
def test_what_takes_no_part_gets_zero_whatever_its_task_holds(E):
    """Padding and a token all at -inf, in a task with a NaN logit and in one whose losses have infinite weights."""
    T, N, k = 3, 70, 2
    x, idx, dloss = _inputs(T, N, E, k, seed=19)
    mask = torch.ones(T, N, dtype=torch.uint8)
    mask[:, 40:] = 0
    x[:, 3] = float("-inf")
    x[0, 5, 2] = float("nan")
    dloss[1] = float("inf")
    o = _run(_problem(T, N, E, k), x.cuda(), idx.cuda(), mask.cuda(), dloss.cuda())
    d = o["dlogits"].cpu()
    assert torch.isnan(o["excess"][0]).any() and not torch.isfinite(d[:2, :3]).all()
    assert torch.all(d[:, 40:] == 0) and torch.all(d[:, 3] == 0)
    _check({n: v[2:] for n, v in o.items()}, x[2:], idx[2:], mask[2:], dloss[2:])
