"""vmoe_block_norm_bwd with infinities, on a GB300: a sum of one infinity and numbers is that infinity, and what
does not depend on a value is a number whatever that value is.  Signs are exact; numbers within half a step of
the type and 4e-6 of the value (three products in fp32)."""
import pytest
import torch

import paper_2608_16188_gb300 as vm

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__
    __graft_entry__.build()


def _run(dtype, N, d, post, y, dz, gate, post_w=None, post_b=None):
    """z = x + gate * (norm of) y, without a norm ahead of the next layer, and its gradients."""
    T = y.shape[0]
    p, cfg = vm.problem(T, N, d, 8, 1, 1, 1.0, dtype), vm.norm_config(post=post, eps=1e-5)
    x, z, dx, dy = (torch.full_like(y, 0.5) for _ in range(4))
    stat = torch.empty(T, N, 2, device="cuda") if post else None
    g = {n: None if v is None else torch.full_like(v, float("nan")) for n, v in (("w", post_w), ("b", post_b), ("g", gate))}
    ws = torch.empty(vm.vmoe_block_norm_bwd_workspace_size(p), dtype=torch.uint8, device="cuda")
    vm.vmoe_block_norm(p, cfg, x, y, post_w, post_b, gate, None, None, z, None, stat)
    vm.vmoe_block_norm_bwd(p, cfg, y, None, stat, None, post_w, post_b, gate, None, dz, None, dx, dy, g["w"], g["b"], g["g"], None,
                           None, ws)
    return dx, dy, g


def _data(dtype, N, d, seed=1):
    gen = torch.Generator().manual_seed(seed + N + d)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    y, dz = (torch.randn(2, N, d, generator=gen).to(dt).cuda() for _ in range(2))
    gate = (0.5 + torch.rand(2, d, generator=gen)).cuda()
    return y, dz, gate


SIZES = [(1, 8), (5, 64), (7, 200), (101, 768), (301, 1000), (9, 1304)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,d", SIZES)
@pytest.mark.parametrize("form", ["no_norm", "no_bias", "zero_bias", "zero_weight"])
def test_an_infinite_gradient_reaches_the_gate(N, d, dtype, form):
    """dgate = sum dzt w, one term of it infinite: the infinity with the sign of w there."""
    y, dz, gate = _data(dtype, N, d)
    dz[1, N - 1, 3] = float("inf")
    post = form != "no_norm"
    one = torch.ones_like(gate)
    post_w = None if not post else 0 * one if form == "zero_weight" else one
    post_b = {"zero_bias": 0 * one, "zero_weight": -one}.get(form)
    _, _, g = _run(dtype, N, d, post, y, dz, gate, post_w, post_b)
    row = y[1, N - 1].double()
    sign = -1.0 if form == "zero_weight" else float(torch.sign((row - row.mean() if post else row)[3]))
    got = g["g"].cpu()
    assert sign != 0 and float(got[1, 3]) == sign * float("inf"), got[1, 3]
    got[1, 3] = 0.0
    assert torch.isfinite(got).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,d", SIZES)
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_without_a_norm_the_gradient_of_the_branch_does_not_depend_on_it(N, d, dtype, value):
    """dy = gate dz and dx = dz, whatever y holds; dgate = sum dz y has it in its column alone."""
    y, dz, gate = _data(dtype, N, d, seed=5)
    y[0, N // 2, 5] = value
    dx, dy, g = _run(dtype, N, d, False, y, dz, gate)
    assert torch.equal(dx, dz)
    ref = gate[:, None, :].double() * dz.double()
    assert ((dy.double() - ref).abs() <= (HALF[dtype] + 4e-6) * ref.abs()).all()
    bad = ~torch.isfinite(g["g"].cpu())
    assert bad[0, 5] and int(bad.sum()) == 1
