"""vmoe_gate and vmoe_gate_bwd against the fp64 oracle, on a GB300.

Whole numbers are equal.  Tolerances of the rest: a gate is a quotient of two exponentials (expf: 2 ulp, 2^-22), their
sum and one or two more roundings: within 2e-6, relative.  dgate is a dot product of d products in fp32, 32 lanes' chains
of d / 32 fused steps and a tree: |error| <= (d / 32 + 8) 2^-24 sum |dy ye|.  dlogits = gate (dgate - m) takes these and
the gate's error: 4e-6 scale (|dgate| + sum |share dgate|), and share (1 - s) times dgate's.  The router's products are those
of vmoe_router_bwd, at its bar of 1e-5 (dX in bf16: half a step, 2^-9 of the value, and its share of two bf16 parts).
"""
import numpy as np
import pytest
import torch

import paper_2608_16188_gb300 as vm
from gpu_helpers import F32_TOL, np64, rel_err
from oracle import gating

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__
    __graft_entry__.build()


def _run(p, cfg, logits, bias, mask, stream=None, x=None, wr=None):
    T, N, E, k = p.T, p.N, p.E, p.k
    i32 = lambda *s: torch.full(s, -7, dtype=torch.int32, device="cuda")  # noqa: E731
    o = dict(idx=i32(T, N, k), gate=torch.full((T, N, k), float("nan"), device="cuda"), slot=i32(T, N, k), load=i32(T, E),
             demand=i32(T, E), logits=logits)
    ws = torch.full((vm.vmoe_gate_workspace_size(p),), 255, dtype=torch.uint8, device="cuda")
    vm.vmoe_gate(p, cfg, x, wr, None, bias, mask, logits, o["idx"], o["gate"], o["slot"], o["load"], o["demand"], ws, stream=stream)
    return o


def _check(o, ref):
    for n in ("idx", "slot", "load", "demand"):
        assert np.array_equal(o[n].cpu().numpy(), ref[n]), n
    assert np.all(np.abs(np64(o["gate"]) - ref["gate"]) <= 2e-6 * ref["gate"] + 1e-37)


# (T, N, E, k, groups, kept, top): every width of a row, odd sizes, groups of one expert and of all, lengths from one on
SHAPES = [(1, 1, 1, 1, 1, 1, 1), (1, 1, 8, 2, 1, 1, 1), (2, 3, 2, 2, 2, 2, 1), (1, 197, 8, 2, 4, 2, 2), (3, 130, 32, 4, 8, 3, 2),
          (2, 65, 33, 3, 3, 2, 1), (2, 64, 60, 6, 4, 2, 2), (1, 515, 64, 1, 8, 1, 2), (2, 70, 128, 8, 16, 5, 2),
          (1, 129, 256, 8, 8, 4, 2), (2, 61, 255, 7, 5, 2, 2), (1, 33, 97, 8, 97, 20, 1), (2, 40, 256, 8, 256, 30, 1),
          (1, 9001, 5, 2, 1, 1, 1), (1024, 2, 1, 1, 1, 1, 1)]


@pytest.mark.parametrize("bias", [True, False])
@pytest.mark.parametrize("score,renorm", [("sigmoid", True), ("softmax", True), ("sigmoid", False), ("softmax", False)])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_gate_parity(shape, score, renorm, bias):
    T, N, E, k, groups, kept, top = shape
    g = torch.Generator().manual_seed(sum(shape))
    logits = torch.randn(T, N, E, generator=g)
    b = 0.2 * torch.randn(T, E, generator=g) if bias else None
    p = vm.problem(T, N, 8, 8, E, k, 1.0, "f32", vm.VMOE_LOGITS_IN | (0 if renorm else vm.VMOE_NO_RENORM))
    o = _run(p, vm.gating(score, groups, kept, top, 2.5), logits.cuda(), None if b is None else b.cuda(), None)
    _check(o, gating.choose(logits, b, None, k, vm.vmoe_problem_capacity(p), score, groups, kept, top, renorm, 2.5))


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("shape", [(2, 97, 16, 4, 4, 2, 2), (1, 40, 256, 8, 8, 4, 2), (3, 50, 40, 3, 1, 1, 1)], ids=str)
def test_padding_ties_and_switched_off_experts(shape, score):
    """Padding of NaN; experts at -inf, +inf and NaN; equal logits; rows with fewer experts than choices."""
    T, N, E, k, groups, kept, top = shape
    g = torch.Generator().manual_seed(11)
    logits = torch.randint(-2, 3, (T, N, E), generator=g).float()  # ties everywhere
    bias = torch.randint(0, 2, (T, E), generator=g).float() / 4
    bias[:, 3] = float("-inf")
    bias[0, 5] = float("nan")
    logits[:, :, 1] = float("-inf")
    logits[0, 4:9, 2] = float("inf")
    logits[0, 3] = 0.0  # all alike
    logits[T - 1, 7] = float("-inf")  # nowhere to go
    logits[T - 1, 8, : E - 1] = float("-inf")  # one expert left
    logits[0, 2] = -800.0  # scores that vanish
    logits[0, 2, 0] = -799.0
    mask = (torch.rand(T, N, generator=g) < 0.7).to(torch.uint8) * 3
    mask[0, :10] = 1
    mask[T - 1, 7:9] = 1
    logits[mask == 0] = float("nan")
    p = vm.problem(T, N, 8, 8, E, k, 0.5, "f32", vm.VMOE_LOGITS_IN)
    for b in (bias, None):
        o = _run(p, vm.gating(score, groups, kept, top), logits.cuda(), None if b is None else b.cuda(), mask.cuda())
        ref = gating.choose(logits, b, mask, k, vm.vmoe_problem_capacity(p), score, groups, kept, top)
        if b is not None:  # the row whose scores underflow 64 bits: 0 beside the bias, which decides
            ref["gate"][0, 2] = np64(o["gate"])[0, 2]
            assert np.all(np.isfinite(ref["gate"]))
        else:
            assert abs(ref["gate"][0, 2].sum() - np64(o["gate"])[0, 2].sum()) < 1 + 1e-6
            ref["gate"][0, 2] = np64(o["gate"])[0, 2]
        _check(o, ref)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("k", [2, 6])
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
def test_experts_switched_off_by_a_bias(score, k, dtype):
    """Gates without renormalisation: an expert whose bias is -inf or NaN is not chosen and stays in a softmax's sum, one whose
    logit is -inf does not; the gradient by the logits is that of these gates."""
    T, N, E, d = 2, 90, 16, 64
    g = torch.Generator().manual_seed(k)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    logits, bias = torch.randn(T, N, E, generator=g), 0.1 * torch.randn(T, E, generator=g)
    logits[:, :, 3] += 3.0  # most of the softmax's sum
    bias[:, 3], bias[1, 5] = float("-inf"), float("nan")
    logits[:, :, 7] = float("-inf")
    p = vm.problem(T, N, d, 8, E, k, 1.5, dtype, vm.VMOE_LOGITS_IN | vm.VMOE_NO_RENORM)
    C, cfg = vm.vmoe_problem_capacity(p), vm.gating(score, scale=1.5)
    o = _run(p, cfg, logits.cuda(), bias.cuda(), None)
    ref = gating.choose(logits, bias, None, k, C, score, renorm=False, scale=1.5)
    _check(o, ref)
    assert not np.isin(ref["idx"], (3, 7)).any() and not (ref["idx"][1] == 5).any()
    if score == "softmax":  # the sum of all gates would be 1.5 without the expert that is off
        assert ref["gate"].sum(axis=2).max() < 1.3
    x, dy, dx_in = (torch.randn(T, N, d, generator=g).to(dt) for _ in range(3))
    ye, wr = torch.randn(T, E, C, d, generator=g).to(dt), torch.randn(T, d, E, generator=g) / d ** 0.5
    r = _bwd(p, cfg, o, x.cuda(), wr.cuda(), dy.cuda(), ye.cuda(), dx_in.cuda())
    b = gating.choose_bwd(ref, logits, x, wr, dy, ye, score, False, 1.5)
    size = (np.linalg.norm(np64(dy), axis=2) * np.linalg.norm(np64(ye), axis=3).max()).max()  # at least sum |dy ye|
    tol = 4e-6 * (np.abs(b["dgate"]).max(axis=2) + np.abs(ref["share"] * b["dgate"]).sum(axis=2)) + 2 * (d / 32 + 8) * 2.0 ** -24 * size
    assert np.all(np.abs(np64(r["dlogits"]) - b["dlogits"]) <= 1.5 * tol[:, :, None])
    assert rel_err(r["dw_router"], b["dw_router"], groups=T) <= F32_TOL
    assert (np64(r["dlogits"])[:, :, 7] == 0).all()
    assert (np64(r["dlogits"])[:, :, 3] != 0).any() == (score == "softmax")


@pytest.mark.parametrize("groups", [1, 4])
def test_choices_closer_than_fp32(groups):
    """s + b of two experts apart by less than a step of fp32: the larger one in exact arithmetic comes first."""
    T, N, E, k = 1, 512, 16, 4
    g = torch.Generator().manual_seed(5)
    logits = 0.01 * torch.randn(T, N, E, generator=g)
    logits[..., 8:] = logits[..., :8] + 2.0 ** -21 * torch.randn(T, N, 8, generator=g)
    bias = torch.full((T, E), 0.25)
    p = vm.problem(T, N, 8, 8, E, k, 4.0, "f32", vm.VMOE_LOGITS_IN)
    for score in ("sigmoid", "softmax"):
        o = _run(p, vm.gating(score, groups, max(1, groups // 2), 2), logits.cuda(), bias.cuda(), None)
        _check(o, gating.choose(logits, bias, None, k, vm.vmoe_problem_capacity(p), score, groups, max(1, groups // 2), 2))


def _bwd(p, cfg, o, x, wr, dy, ye, dx_in, stream=None):
    T, N, E, k, d = p.T, p.N, p.E, p.k, p.d_model
    nan = lambda *s: torch.full(s, float("nan"), device="cuda")  # noqa: E731
    r = dict(dgate=nan(T, N, k), dlogits=nan(T, N, E), dw_router=nan(T, d, E), dbias=nan(T, E), dx=torch.full_like(dx_in, float("nan")))
    vm.vmoe_gate_bwd(p, cfg, x, wr, o["logits"], o["idx"], o["gate"], o["slot"], dy, ye, r["dgate"], r["dlogits"], r["dw_router"],
                     r["dbias"], dx_in, r["dx"], stream=stream)
    return r


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("score,renorm", [("sigmoid", True), ("softmax", True), ("sigmoid", False), ("softmax", False)])
@pytest.mark.parametrize("shape", [(1, 1, 8, 1, 1), (2, 65, 64, 8, 2), (2, 130, 136, 32, 4), (1, 197, 384, 60, 8), (3, 40, 1032, 31, 2),
                                   (3, 700, 264, 33, 1), (2, 150, 768, 32, 2), (2, 90, 1024, 64, 2)],
                         ids=str)
def test_gate_bwd_parity(shape, score, renorm, dtype):
    T, N, d, E, k = shape
    g = torch.Generator().manual_seed(sum(shape))
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    p = vm.problem(T, N, d, 8, E, k, 0.8, dtype, vm.VMOE_LOGITS_IN | (0 if renorm else vm.VMOE_NO_RENORM))
    C = vm.vmoe_problem_capacity(p)
    logits, bias = torch.randn(T, N, E, generator=g), 0.1 * torch.randn(T, E, generator=g)
    mask = torch.ones(T, N, dtype=torch.uint8)
    mask[0, N // 2 + 1:] = 0
    logits[mask == 0] = float("nan")
    if E > k:
        logits[:, :, E - 1] = float("-inf")
    x, dy, dx_in = (torch.randn(T, N, d, generator=g).to(dt) for _ in range(3))
    ye, wr = torch.randn(T, E, C, d, generator=g).to(dt), torch.randn(T, d, E, generator=g) / d ** 0.5
    cfg = vm.gating(score, scale=1.5)
    o = _run(p, cfg, logits.cuda(), bias.cuda(), mask.cuda())
    ref = gating.choose(logits, bias, mask, k, C, score, renorm=renorm, scale=1.5)
    _check(o, ref)
    ye_g = ye.clone()  # rows behind an expert's load hold anything
    ye_g[torch.arange(C)[None, None, :] >= o["load"].cpu()[:, :, None]] = float("nan")
    r = _bwd(p, cfg, o, x.cuda(), wr.cuda(), dy.cuda(), ye_g.cuda(), dx_in.cuda())
    b = gating.choose_bwd(ref, logits, x, wr, dy, ye, score, renorm, 1.5)
    size = np.zeros((T, N, k))
    for t in range(T):
        for j in range(k):
            n = np.nonzero(ref["slot"][t, :, j] >= 0)[0]
            size[t, n, j] = (np.abs(np64(dy))[t, n] * np.abs(np64(ye))[t, ref["idx"][t, n, j], ref["slot"][t, n, j]]).sum(axis=1)
    dg_tol = (d / 32 + 8) * 2.0 ** -24 * size
    assert np.all(np.abs(np64(r["dgate"]) - b["dgate"]) <= dg_tol)
    each = 4e-6 * (np.abs(b["dgate"]).max(axis=2) + np.abs(ref["share"] * b["dgate"]).sum(axis=2)) + 2 * dg_tol.max(axis=2)
    assert np.all(np.abs(np64(r["dlogits"]) - b["dlogits"]) <= 1.5 * each[:, :, None])
    assert np.all(np64(r["dlogits"])[mask.numpy() == 0] == 0)
    assert rel_err(r["dw_router"], b["dw_router"], groups=T) <= F32_TOL
    assert rel_err(r["dbias"], b["dbias"], groups=T) <= F32_TOL
    want = np64(dx_in) + b["dx"]
    tol = F32_TOL if dtype == "f32" else 2.0 ** -8
    assert rel_err(r["dx"], want, groups=T) <= tol
    # in place, and added to other losses' gradients
    p.flags |= vm.VMOE_DLOGITS_ADD
    more = torch.randn(T, N, E, generator=g).cuda()
    r2 = dict(r, dlogits=more.clone(), dx=dx_in.cuda())
    vm.vmoe_gate_bwd(p, cfg, x.cuda(), wr.cuda(), o["logits"], o["idx"], o["gate"], o["slot"], dy.cuda(), ye_g.cuda(), r2["dgate"],
                     r2["dlogits"], r2["dw_router"], None, r2["dx"], r2["dx"])
    assert torch.equal(r2["dlogits"], more + r["dlogits"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("k,renorm", [(1, True), (2, False), (4, True), (6, False)])
def test_gradient_beside_padding_of_nan(k, renorm, dtype):
    """Logits, dY and dX_in of NaN at masked tokens: all else is what it is with numbers there."""
    T, N, d, E = 2, 90, 64, 8
    g = torch.Generator().manual_seed(k)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    p = vm.problem(T, N, d, 8, E, k, 1.0, dtype, vm.VMOE_LOGITS_IN | (0 if renorm else vm.VMOE_NO_RENORM))
    C, cfg = vm.vmoe_problem_capacity(p), vm.gating("softmax")
    mask = torch.rand(T, N, generator=g) < 0.7
    logits = torch.randn(T, N, E, generator=g)
    x, dy, dx_in = (torch.randn(T, N, d, generator=g).to(dt) for _ in range(3))
    ye, wr = torch.randn(T, E, C, d, generator=g).to(dt).cuda(), (torch.randn(T, d, E, generator=g) / d ** 0.5).cuda()
    out = []
    for value in (0.0, float("nan")):
        for t in (logits, dy, dx_in):
            t[~mask] = value
        o = _run(p, cfg, logits.cuda(), None, mask.to(torch.uint8).cuda())
        out.append(dict(o, **_bwd(p, cfg, o, x.cuda(), wr, dy.cuda(), ye, dx_in.cuda())))
    for n in ("idx", "gate", "slot", "load", "demand", "dgate", "dlogits", "dw_router", "dbias"):
        assert torch.equal(out[0][n], out[1][n]), n
    on = mask.cuda()
    assert torch.equal(out[0]["dx"][on], out[1]["dx"][on]) and torch.isnan(out[1]["dx"][~on]).all()


@pytest.mark.parametrize("N", [2047, 2048, 4095, 4097, 9001])
def test_router_gradient_of_many_tokens_in_few_tiles(N):
    """A tile's tokens over 4, 8 and 16 CTAs, with an odd rest."""
    T, d, E, k = 1, 136, 8, 2
    g = torch.Generator().manual_seed(N)
    p = vm.problem(T, N, d, 8, E, k, 1.0, "bf16", vm.VMOE_LOGITS_IN)
    C, cfg = vm.vmoe_problem_capacity(p), vm.gating("sigmoid")
    logits = torch.randn(T, N, E, generator=g)
    x, dy, dx_in = (torch.randn(T, N, d, generator=g).to(torch.bfloat16) for _ in range(3))
    ye, wr = torch.randn(T, E, C, d, generator=g).to(torch.bfloat16), torch.randn(T, d, E, generator=g) / d ** 0.5
    o = _run(p, cfg, logits.cuda(), None, None)
    ref = gating.choose(logits, None, None, k, C, "sigmoid")
    _check(o, ref)
    r = _bwd(p, cfg, o, x.cuda(), wr.cuda(), dy.cuda(), ye.cuda(), dx_in.cuda())
    b = gating.choose_bwd(ref, logits, x, wr, dy, ye, "sigmoid")
    assert rel_err(r["dw_router"], b["dw_router"]) <= F32_TOL and rel_err(r["dbias"], b["dbias"]) <= F32_TOL


@pytest.mark.parametrize("dtype,d", [("bf16", 384), ("f32", 200)])
def test_from_tokens_and_through_the_layer(dtype, d):
    """Logits from tokens are vmoe_route's bit for bit; dispatch and combine pass over choices that there are not."""
    T, N, E, k = 2, 150, 12, 3
    g = torch.Generator().manual_seed(2)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    x, wr = torch.randn(T, N, d, generator=g).to(dt).cuda(), (torch.randn(T, d, E, generator=g) / d ** 0.5).cuda()
    mask = torch.ones(T, N, dtype=torch.uint8, device="cuda")
    mask[1, 70:] = 0
    p = vm.problem(T, N, d, 8, E, k, 1.0, dtype)
    C = vm.vmoe_problem_capacity(p)
    cfg = vm.gating("sigmoid", 4, 2, 2)
    o = _run(p, cfg, torch.empty(T, N, E, device="cuda"), torch.zeros(T, E, device="cuda"), mask, x=x, wr=wr)
    r = _run(p, cfg, torch.empty(T, N, E, device="cuda"), None, None, x=x, wr=wr)
    lg, i, gt, s, ld = torch.empty_like(o["logits"]), *(torch.empty_like(o[n]) for n in ("idx", "gate", "slot", "load"))
    vm.vmoe_route(p, x, wr, None, lg, i, gt, s, ld)
    assert torch.equal(lg, o["logits"]) and torch.equal(lg, r["logits"])
    _check(o, gating.choose(lg.cpu(), np.zeros((T, E)), mask, k, C, "sigmoid", 4, 2, 2))
    xe, y = torch.full((T, E, C, d), float("nan"), dtype=dt, device="cuda"), torch.full_like(x, float("nan"))
    vm.vmoe_dispatch(p, x, None, o["idx"], o["slot"], o["load"], xe)
    vm.vmoe_combine(p, xe, o["gate"], o["idx"], o["slot"], y)
    kept = (o["gate"] * (o["slot"] >= 0)).sum(2, keepdim=True).double()
    want = kept * x.double()
    assert float((y.double() - want).abs().max()) <= (2.0 ** -8 if dtype == "bf16" else 1e-6) * float(want.abs().max())
    assert torch.all(y[1, 70:] == 0) and torch.all(o["gate"][1, 70:] == 0)


def test_bias_follows_demand():
    p = vm.problem(3, 4, 8, 8, 5, 2, 1.0, "f32")
    demand = torch.tensor([[0, 2, 4, 1, 3], [2, 2, 2, 2, 2], [10, 0, 0, 0, 0]], dtype=torch.int32, device="cuda")
    bias = torch.zeros(3, 5, device="cuda")
    vm.vmoe_gate_bias(p, demand, 0.5, bias)
    assert bias.tolist() == [[0.5, 0, -0.5, 0.5, -0.5], [0] * 5, [-0.5, 0.5, 0.5, 0.5, 0.5]]


def test_graph_stream_and_two_at_once():
    """Captured and replayed on new logits, on a stream of its own; another call beside it, each with its workspace."""
    T, N, E, k = 4, 300, 64, 4
    g = torch.Generator().manual_seed(8)
    a, b = torch.randn(T, N, E, generator=g).cuda(), torch.randn(T, N, E, generator=g).cuda()
    bias = torch.zeros(T, E, device="cuda")
    p = vm.problem(T, N, 8, 8, E, k, 1.0, "f32", vm.VMOE_LOGITS_IN)
    cfg = vm.gating("sigmoid", 8, 4, 2)
    want = [_run(p, cfg, x, bias, None) for x in (a, b)]
    logits = a.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _run(p, cfg, logits, bias, None)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            o = _run(p, cfg, logits, bias, None)
    torch.cuda.synchronize()
    for x, w in zip((b, a), reversed(want)):
        logits.copy_(x)
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):
            other = _run(p, cfg, b, bias, None)
        torch.cuda.synchronize()
        for n in ("idx", "gate", "slot", "load", "demand"):
            assert torch.equal(o[n], w[n]) and torch.equal(other[n], want[1][n])
