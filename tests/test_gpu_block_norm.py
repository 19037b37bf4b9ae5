"""vmoe_block_norm and its backward against the fp64 oracle, on a GB300.

Stage by stage, as for the other calls: u and the backward are compared given the z that the GPU stored.
Tolerances, per element:
  a stored output is one rounding of its fp32 value: half a step, eps / 2 of itself (bf16 2^-8, fp32 2^-24);
  the fp32 value: means and variances are sums of d <= 8192 values, 8 to 32 a thread and then in a tree, so
  within 48 x 2^-24 = 3e-6 of the sum of magnitudes; (v - mean) rstd inherits that, relative to the row's
  largest normalised value; 1e-5 of the row's largest magnitude (times its parameters) covers both statistics;
  a parameter's gradient: terms within 1e-5, summed in runs: 1.2e-5 of the terms' magnitudes.
"""
import numpy as np
import pytest
import torch

import paper_2608_16188_gb300 as vm
from gpu_helpers import np64
from oracle import training as tr

pytestmark = pytest.mark.gpu

EPS = 1e-5
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__
    __graft_entry__.build()


def _make(T, N, d, dtype, part, post, rms, params=True, seed=0):
    g = torch.Generator().manual_seed(seed + T * 1000 + N * 10 + d)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    r = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    s = dict(x=(r(T, N, d) + r(T, 1, d) ** 2).to(dt), dz=r(T, N, d).to(dt), y=None, du=None)
    for n in ("post_w", "post_b", "gate", "pre_w", "pre_b"):
        s[n] = None
    if part != "pre":
        s["y"] = (2 * r(T, N, d) + 0.3).to(dt)
        if params:
            s["gate"] = 0.5 + 0.2 * r(T, d)
            if post:
                s["post_w"] = 1 + 0.1 * r(T, d)
                s["post_b"] = None if rms else 0.1 * r(T, d)
    if part != "post":
        s["du"] = r(T, N, d).to(dt)
        if params:
            s["pre_w"] = 1 + 0.1 * r(T, d)
            s["pre_b"] = None if rms else 0.1 * r(T, d)
    return {n: None if v is None else v.cuda() for n, v in s.items()}


def _run(s, dtype, part, post, rms, rho, stream=None, p=None):
    T, N, d = s["x"].shape
    p = vm.problem(T, N, d, 8, 1, 1, 1.0, dtype)
    cfg = vm.norm_config(rms=rms, post=post, eps=EPS, residual_scale=rho)
    bad = lambda ref, have=True: torch.full_like(ref, float("nan")) if have and ref is not None else None  # noqa: E731
    stat = lambda have: torch.full((T, N, 2), float("nan"), device="cuda") if have else None  # noqa: E731
    o = dict(z=bad(s["x"], part != "pre"), u=bad(s["x"], part != "post"))
    ps, qs = stat(part != "pre" and post), stat(part != "post")
    vm.vmoe_block_norm(p, cfg, s["x"], s["y"], s["post_w"], s["post_b"], s["gate"], s["pre_w"], s["pre_b"], o["z"],
                       o["u"], ps, qs, stream=stream)
    o["dx"], o["dy"] = bad(s["x"]), bad(s["y"])
    for n in ("post_w", "post_b", "gate", "pre_w"):
        o["d" + n] = bad(s[n])
    o["dpre_b"] = bad(s["pre_w"])
    ws = torch.full((vm.vmoe_block_norm_bwd_workspace_size(p),), 255, dtype=torch.uint8, device="cuda")
    vm.vmoe_block_norm_bwd(p, cfg, s["y"], s["x"] if part == "pre" else o["z"], ps, qs, s["post_w"], s["post_b"], s["gate"],
                           s["pre_w"], s["dz"], s["du"], o["dx"], o["dy"], o["dpost_w"], o["dpost_b"], o["dgate"],
                           o["dpre_w"], o["dpre_b"], ws, stream=stream)
    return o


def _near(name, got, ref, half):
    got, ref = np64(got), np.asarray(ref)
    tol = half * np.abs(ref) + 1e-5 * np.abs(ref).max(axis=2, keepdims=True) + 1e-30
    bad = np.abs(got - ref) > tol
    assert not bad.any(), (name, int(bad.sum()), float((np.abs(got - ref) / tol).max()))


def _check(s, o, dtype, part, post, rms, rho):
    half = HALF[dtype]
    if part != "pre":
        _near("z", o["z"], tr.block_z(s["x"], s["y"], s["post_w"], s["post_b"], s["gate"], rho, rms, post, EPS), half)
    z = s["x"] if part == "pre" else o["z"]
    if part != "post":
        _near("u", o["u"], tr.norm(np64(z), s["pre_w"], s["pre_b"], rms, EPS), half)
    ref, mag = tr.block_bwd(s["y"], z, s["post_w"], s["post_b"], s["gate"], s["pre_w"], s["dz"], s["du"], rho, rms, post, EPS)
    for n in ("dx", "dy"):
        if o[n] is not None:
            _near(n, o[n], ref[n], half)
    for n in ("dpost_w", "dpost_b", "dgate", "dpre_w", "dpre_b"):
        if o.get(n) is not None:
            err = np.abs(np64(o[n]) - ref[n])
            assert np.all(err <= 1.2e-5 * mag[n] + 1e-30), (n, float((err / (mag[n] + 1e-30)).max()))


# widths around each form's border (8 lanes a row up to 64 channels, 16 up to 128, a warp for each 256, 8192 the
# most), odd counts of tokens
SHAPES = [(1, 1, 8), (2, 3, 16), (1, 197, 384), (3, 50, 248), (2, 33, 264), (2, 40, 512), (2, 65, 768), (3, 77, 1000),
          (1, 130, 1024), (2, 9, 1032), (1, 21, 2048), (2, 5, 2056), (1, 13, 4104), (1, 3, 8192), (5, 700, 96),
          (7, 5, 40), (4, 37, 64), (2, 611, 72), (3, 211, 128), (2, 90, 136)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_block_norm_parity(shape, dtype):
    s = _make(*shape, dtype, "both", True, False)
    _check(s, _run(s, dtype, "both", True, False, 1.25), dtype, "both", True, False, 1.25)


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("part", ["pre", "post", "both"])
@pytest.mark.parametrize("params", [False, True])
def test_every_part_and_missing_parameters(rms, post, part, params):
    for dtype, shape in (("bf16", (2, 37, 200)), ("f32", (2, 19, 1536))):
        s = _make(*shape, dtype, part, post, rms, params)
        _check(s, _run(s, dtype, part, post, rms, 0.75), dtype, part, post, rms, 0.75)


def test_constant_and_zero_rows_are_finite():
    """A row without variance: rstd is 1 / sqrt(eps)."""
    s = _make(1, 4, 64, "f32", "both", True, False)
    s["y"][0, 0] = 3.0
    s["y"][0, 1] = 0.0
    s["x"][0, 2] = 0.0
    s["y"][0, 2] = 0.0
    o = _run(s, "f32", "both", True, False, 1.0)
    assert all(torch.isfinite(v).all() for v in o.values() if v is not None)
    _check(s, o, "f32", "both", True, False, 1.0)


def test_a_large_mean_keeps_its_variance():
    """Mean 1000, deviation 1: the squares' difference would keep 2 digits.  (v - mean) loses 1000 x 2^-24 = 6e-5
    of the deviation, the same in the oracle's input: the mean itself is within 1000 x 3e-6 / 32 (its error is a
    sum's), so normalised values within 1e-3 absolute."""
    s = _make(1, 8, 768, "f32", "pre", False, False, params=False)
    s["x"] = s["x"] * 0.5 + 1000.0
    p = vm.problem(1, 8, 768, 8, 1, 1, 1.0, "f32")
    u = torch.empty_like(s["x"])
    vm.vmoe_block_norm(p, vm.norm_config(eps=EPS), s["x"], None, None, None, None, None, None, None, u)
    assert np.max(np.abs(np64(u) - tr.norm(np64(s["x"]), None, None, False, EPS))) < 1e-3


def test_nan_stays_in_its_row():
    s = _make(2, 6, 256, "bf16", "both", True, False)
    s["y"][1, 3, 17] = float("nan")
    s["x"][0, 2, 5] = float("inf")
    p = vm.problem(2, 6, 256, 8, 1, 1, 1.0, "bf16")
    z, u = torch.empty_like(s["x"]), torch.empty_like(s["x"])
    vm.vmoe_block_norm(p, vm.norm_config(eps=EPS), s["x"], s["y"], s["post_w"], s["post_b"], s["gate"], s["pre_w"], s["pre_b"], z, u)
    bad = torch.zeros(2, 6, dtype=torch.bool, device="cuda")
    bad[1, 3] = bad[0, 2] = True
    assert torch.equal(torch.isnan(u).any(dim=2), bad) and torch.isfinite(u[~bad]).all() and torch.isfinite(z[~bad]).all()


def test_in_place_streams_graphs_and_determinism():
    """z over x and dx over dz give the same values; another stream and a replayed graph too."""
    T, N, d = 3, 210, 384
    s = _make(T, N, d, "bf16", "both", True, False)
    a = _run(s, "bf16", "both", True, False, 1.1)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    b = _run(s, "bf16", "both", True, False, 1.1, stream=st)
    torch.cuda.synchronize()
    assert all(v is None or torch.equal(v, b[n]) for n, v in a.items())
    p, cfg = vm.problem(T, N, d, 8, 1, 1, 1.0, "bf16"), vm.norm_config(eps=EPS, residual_scale=1.1)
    x, dz = s["x"].clone(), s["dz"].clone()
    o = {n: torch.empty_like(v) for n, v in a.items() if v is not None}
    ps, qs = torch.empty(T, N, 2, device="cuda"), torch.empty(T, N, 2, device="cuda")
    ws = torch.empty(vm.vmoe_block_norm_bwd_workspace_size(p), dtype=torch.uint8, device="cuda")

    def both():
        vm.vmoe_block_norm(p, cfg, x, s["y"], s["post_w"], s["post_b"], s["gate"], s["pre_w"], s["pre_b"], x, o["u"], ps, qs)
        vm.vmoe_block_norm_bwd(p, cfg, s["y"], x, ps, qs, s["post_w"], s["post_b"], s["gate"], s["pre_w"], dz, s["du"], dz,
                               o["dy"], o["dpost_w"], o["dpost_b"], o["dgate"], o["dpre_w"], o["dpre_b"], ws)

    both()
    torch.cuda.synchronize()
    o["z"], o["dx"] = x.clone(), dz.clone()
    assert all(torch.equal(o[n], a[n]) for n in o)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(2):
        x.copy_(s["x"])
        dz.copy_(s["dz"])
        graph.replay()
        torch.cuda.synchronize()
        o["z"], o["dx"] = x, dz
        assert all(torch.equal(o[n], a[n]) for n in o)


def test_no_dz_and_no_parameter_gradients():
    s = _make(2, 20, 96, "f32", "both", True, False)
    s["dz"].zero_()
    a = _run(s, "f32", "both", True, False, 1.0)
    p, cfg = vm.problem(2, 20, 96, 8, 1, 1, 1.0, "f32"), vm.norm_config(eps=EPS)
    ps, qs = torch.empty(2, 20, 2, device="cuda"), torch.empty(2, 20, 2, device="cuda")
    z, u, dx, dy = (torch.empty_like(s["x"]) for _ in range(4))
    ws = torch.empty(vm.vmoe_block_norm_bwd_workspace_size(p), dtype=torch.uint8, device="cuda")
    vm.vmoe_block_norm(p, cfg, s["x"], s["y"], s["post_w"], s["post_b"], s["gate"], s["pre_w"], s["pre_b"], z, u, ps, qs)
    vm.vmoe_block_norm_bwd(p, cfg, s["y"], z, ps, qs, s["post_w"], s["post_b"], s["gate"], s["pre_w"], None, s["du"], dx, dy,
                           None, None, None, None, None, ws)
    torch.cuda.synchronize()
    assert torch.equal(dx, a["dx"]) and torch.equal(dy, a["dy"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,d", [(1, 8), (5, 64), (3, 104), (7, 200), (1, 256), (33, 512), (101, 768), (5, 1024), (301, 1000), (3, 1304)])
def test_an_infinite_gradient_in_the_last_token_stays_in_its_column(N, d, dtype):
    """Sums of one infinity and numbers are that infinity, in its column alone: nothing is added for rows of a
    step that lie behind the last token."""
    for part, grad, name in (("post", "dz", "dpost_b"), ("pre", "du", "dpre_b")):
        s = _make(2, N, d, dtype, part, True, False, seed=5)
        s[grad][1, N - 1, 3] = float("inf")
        o = _run(s, dtype, part, True, False, 1.0)
        got = o[name].cpu()
        assert got[1, 3] == float("inf"), (part, got[1, 3])
        got[1, 3] = 0.0
        assert torch.isfinite(got).all(), part
