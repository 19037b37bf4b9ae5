"""vmoe_adamw against the fp64 oracle, on a GB300.

Tolerances.  m and v are two roundings of a sum of two terms, and b1, b2, 1 - b1, 1 - b2 one each:
4 x 2^-24 of the terms' magnitudes.  The update passes expm1, two approximate reciprocals and roots
(2^-22 each) and half a dozen roundings: 4e-6 of itself, next to 2 x 2^-24 of the parameter.  bf16
parameters: 2^-8 more.  8-bit moments: the scale is a maximum, 2^-21; an element is the oracle's neighbour
unless the random number lies near its border, and never further than the next one.  Near: the value, at most
16 steps, is within 1e-6 of itself, 2e-4 steps with a margin of ten, and an m in which the two terms cancel
is within 4 x 2^-24 of the terms, not of itself: that, over the scale and the step, is added.
"""
import numpy as np
import pytest
import torch

import paper_2608_16188_gb300 as vm
from gpu_helpers import np64
from oracle import training as tr

pytestmark = pytest.mark.gpu

HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8)


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__
    __graft_entry__.build()


def _tensor(n, param="f32", grad="f32", eight=False, master=False, seed=0, decay=0.1, rate=1.0):
    """A tensor with moments of earlier steps, 16 elements of canary behind it in every array."""
    g = torch.Generator().manual_seed(seed * 1000 + n)
    kind = {"f32": torch.float32, "bf16": torch.bfloat16}
    pad = lambda v, dt: torch.cat([v, torch.full((16,), 7.0)]).to(dt).cuda()  # noqa: E731
    r = lambda: torch.randn(n, generator=g)  # noqa: E731
    p, gr = r(), 0.01 * r()
    m, root = 0.003 * r(), 0.01 * (0.1 + torch.rand(n, generator=g))
    t = dict(param=pad(p, kind[param]), grad=pad(gr, kind[grad]), master=pad(p, torch.float32) if master else None)
    if eight:
        nb = (n + 255) // 256
        blocks = lambda v: torch.stack([b.abs().max() for b in v.split(256)]) / 448 if n else torch.zeros(0)  # noqa: E731
        ms, vs = blocks(m), blocks(root)
        per = lambda s: s.repeat_interleave(256)[:n]  # noqa: E731
        t.update(m=pad(m / per(ms), torch.float8_e4m3fn), v=pad(root / per(vs), torch.float8_e4m3fn),
                 m_scale=pad(ms, torch.float32), v_scale=pad(vs, torch.float32))
        assert t["m_scale"].numel() == nb + 16
    else:
        t.update(m=pad(m, torch.float32), v=pad(root * root, torch.float32))
    t.update(lr_scale=rate, weight_decay=decay, n=n)
    return t


def _table(tensors):
    cut = lambda t, k: None if t.get(k) is None else t[k][:(t["n"] + 255) // 256 if "scale" in k else t["n"]]  # noqa: E731
    keys = ("param", "grad", "m", "v", "m_scale", "v_scale", "master")
    return vm.adamw_tensors([dict({k: cut(t, k) for k in keys}, lr_scale=t["lr_scale"], weight_decay=t["weight_decay"])
                             for t in tensors])


def _copy(t):
    return {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in t.items()}


def _expect(t, place, step, seed, gs=1.0, lr=None):
    """Checks tensor `t` (before) against itself (after): returns a function of the tensor after."""
    n = t["n"]
    eight = t.get("m_scale") is not None
    p = np64((t["param"] if t["master"] is None else t["master"])[:n])
    g, m, v = (np64(t[k][:n]) for k in ("grad", "m", "v"))
    if eight:
        per = lambda k: np.repeat(np64(t[k]), 256)[:n]  # noqa: E731
        m, v = m * per("m_scale"), (v * per("v_scale")) ** 2
    h = dict(HYPER, lr=HYPER["lr"] if lr is None else lr)
    rp, rm, rv, upd = tr.adamw(p, g, m, v, step, h["lr"], h["beta1"], h["beta2"], h["eps"], t["lr_scale"], t["weight_decay"], gs)
    u = 2.0 ** -24

    def check(a):
        ptol = 2 * u * np.abs(p) + 4e-6 * upd + 1e-12
        if t["master"] is not None:
            assert np.all(np.abs(np64(a["master"][:n]) - rp) <= ptol)
        half = 2.0 ** -8 if t["param"].dtype == torch.bfloat16 else 0.0
        assert np.all(np.abs(np64(a["param"][:n]) - rp) <= ptol + half * np.abs(rp))
        for k in ("param", "grad", "m", "v", "master", "m_scale", "v_scale"):  # the canaries
            if t.get(k) is not None:
                assert torch.all(a[k][-16:].float() == 7.0), k
        if not eight:
            assert np.all(np.abs(np64(a["m"][:n]) - rm) <= 4 * u * (np.abs(m) + np.abs(g * gs)) + 1e-30)
            assert np.all(np.abs(np64(a["v"][:n]) - rv) <= 5 * u * (v + (g * gs) ** 2) + 1e-30)
            return
        lo, hi = tr.dither_bits(n, place, step, seed)
        for k, val, bits in (("m", rm, lo), ("v", np.sqrt(rv), hi)):
            q, scale, border, grid = tr.e4m3_encode(val, bits)
            got = np64(a[k][:n])
            assert np.all(np.abs(np64(a[k + "_scale"])[:scale.size] - scale) <= 2.0 ** -21 * scale), k
            off = 4 * u * (np.abs(m) + np.abs(g * gs)) if k == "m" else 0.0
            per = np.repeat(scale, 256)[:n]
            far = border > 2e-4 + np.divide(off, per * grid, out=np.zeros(n), where=per > 0)
            assert np.array_equal(got[far], q[far]), (k, int((got[far] != q[far]).sum()))
            assert np.all(np.abs(got - q) <= 2 * grid), k
    return check


def _step(tensors, step=3, seed=5, **kw):
    checks = [_expect(t, i, step, seed, gs=float(kw["grad_scale"]) if kw.get("grad_scale") is not None else 1.0)
              for i, t in enumerate(tensors)]
    vm.vmoe_adamw(_table(tensors), step, seed=seed, **HYPER, **kw)
    torch.cuda.synchronize()
    for c, t in zip(checks, tensors):
        c(t)


KINDS = [("f32", "f32", False), ("bf16", "bf16", False), ("bf16", "bf16", True), ("bf16", "f32", False), ("bf16", "f32", True)]


@pytest.mark.parametrize("n", [1, 7, 8, 9, 255, 256, 257, 2048, 5000, 100003])
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("kind", KINDS, ids=str)
def test_adamw_parity(kind, eight, n):
    param, grad, master = kind
    _step([_tensor(n, param, grad, eight, master)])


def test_many_tensors_of_every_kind():
    """More tensors than one launch takes (380), sizes from 0 on, rates and decays of their own."""
    ts = []
    for i in range(401):
        param, grad, master = KINDS[i % 5]
        n = [0, 1, 300, 17, 513, 256][i % 6]
        ts.append(_tensor(n, param, grad, i % 2 == 0, master, seed=i, decay=0.2 * (i % 3), rate=[1.0, 0.5, 0.0][i % 3]))
    _step(ts, step=11, seed=99, grad_scale=torch.tensor([0.25], device="cuda"))


def test_a_table_of_one_launch_and_a_long_tensor_among_short_ones():
    ts = [_tensor(n, *KINDS[1][:2], True, seed=n) for n in (5, 300000, 3, 70000, 1)]
    _step(ts)


def test_zero_gradients_zero_moments_and_denormals():
    """All-zero blocks stay zero; the smallest moments neither overflow a scale nor become NaN."""
    t = _tensor(768, "bf16", "bf16", True)
    for k in ("grad", "m", "v", "m_scale", "v_scale"):
        t[k][:256 if "scale" not in k else 1] = 0
    t["grad"][256:512] = 1e-38
    t["m"][256:512] = 0
    t["v"][256:512] = 0
    before = _copy(t)
    vm.vmoe_adamw(_table([t]), 1, **HYPER)
    torch.cuda.synchronize()
    for k in ("m", "v"):
        assert torch.all(t[k][:256].float() == 0) and torch.isfinite(t[k].float()).all()
    assert t["m_scale"][0] == 0 and t["v_scale"][0] == 0 and torch.isfinite(t["m_scale"][:3]).all()
    want = before["param"][:256].float() * (1 - HYPER["lr"] * 0.1)
    assert torch.equal(t["param"][:256], want.to(torch.bfloat16))
    assert torch.isfinite(t["param"].float()).all()


@pytest.mark.parametrize("eight", [False, True])
def test_nan_gradients_show_and_stay_in_their_element(eight):
    t = _tensor(1024, "f32", "f32", eight)
    clean = _copy(t)
    t["grad"][700] = float("nan")
    vm.vmoe_adamw(_table([t]), 4, **HYPER)
    vm.vmoe_adamw(_table([clean]), 4, **HYPER)
    torch.cuda.synchronize()
    for k in ("param", "m", "v"):
        bad = torch.isnan(t[k][:1024].float())
        assert bad[700] and int(bad.sum()) == 1, k
    for k in ("param", "m", "v"):
        keep = torch.ones(1024, dtype=torch.bool)
        keep[512:768] = False
        assert torch.equal(t[k][:1024][keep.cuda()].float(), clean[k][:1024][keep.cuda()].float())


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_a_step_with_an_overflowed_scale_is_left_out(bad):
    t = _tensor(3000, "bf16", "bf16", True, True)
    before = _copy(t)
    vm.vmoe_adamw(_table([t]), 2, grad_scale=torch.tensor([bad], device="cuda"), **HYPER)
    torch.cuda.synchronize()
    for k, v in before.items():
        if isinstance(v, torch.Tensor):
            assert torch.equal(v.view(torch.uint8), t[k].view(torch.uint8)), k


def test_a_replayed_graph_counts_its_steps_on_the_device():
    """Five replays with step_dev and lr_dev agree bitwise with five calls, and each rounds with its own hash."""
    t = _tensor(5000, "bf16", "bf16", True, True)
    e = _copy(t)
    step, rate = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.ones(1, device="cuda")
    table = _table([t])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.add_(1)
        vm.vmoe_adamw(table, 0, seed=3, step_dev=step, lr_dev=rate, **HYPER)
    other = _table([e])
    for i in range(1, 6):
        rate.fill_(1.0 / i)
        graph.replay()
        vm.vmoe_adamw(other, i, seed=3, lr_dev=rate, **HYPER)
        torch.cuda.synchronize()
        for k in ("param", "master", "m", "v", "m_scale", "v_scale"):
            assert torch.equal(t[k].view(torch.uint8), e[k].view(torch.uint8)), (i, k)


def test_slow_averages_move_in_8_bits():
    """v decays by 1% a step, an eighth to a sixteenth of an e4m3 step: 60 steps without gradients halve it.
    The mean over 65536 elements: each step's rounding has a variance below step^2 / 4 x the 1/25 of it that is
    at stake, so after 60 steps 0.1 relative an element, 4e-4 of the mean; squares add the variance itself, 1%."""
    n = 65536
    t = _tensor(n, "f32", "f32", True)
    t["grad"].zero_()
    val = lambda: float(((t["v"][:n].float().view(-1, 256) * t["v_scale"][:n // 256, None]) ** 2).double().mean())  # noqa: E731
    start = val()
    table = _table([t])
    for i in range(60):
        vm.vmoe_adamw(table, 10 + i, seed=1, **HYPER)
    assert abs(val() / start / 0.99 ** 60 - 1) < 0.03


def test_streams_and_determinism():
    a = [_tensor(70001, "bf16", "bf16", True), _tensor(4097, "f32", "f32")]
    b = [_copy(t) for t in a]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    vm.vmoe_adamw(_table(a), 7, seed=2, **HYPER)
    vm.vmoe_adamw(_table(b), 7, seed=2, stream=s, **HYPER)
    torch.cuda.synchronize()
    for x, y in zip(a, b):
        for k, v in x.items():
            if isinstance(v, torch.Tensor):
                assert torch.equal(v.view(torch.uint8), y[k].view(torch.uint8)), k
