"""vmoe_router_bwd with VMOE_DLOGITS_ADD: the gradient of further losses by the logits joins the router's, and
dW_r, dbias and dX take the sum.  Against the fp64 oracle given the GPU's routing and expert outputs; the bars
are those of the plain call (fp32 outputs 1e-5 of their RMS, bf16 dX 2e-2)."""
import numpy as np
import pytest
import torch

import oracle
import paper_2608_16188_gb300 as vm
import workloads
from gpu_helpers import BF16_TOL, F32_TOL, np64, problem_of, rel_err, to_dev

pytestmark = pytest.mark.gpu

Config = workloads.Config
CASES = {
    "f32": Config("add_f32", 301, T=2, N=300, d=200, f=96, E=6, k=2, cf=1.0, dtype="f32", bias="drift"),
    "bf16_top2": Config("add_bf16", 302, T=3, N=200, d=384, f=128, E=8, k=2, cf=1.0, dtype="bf16", bias="drift"),
    "bf16_norenorm": Config("add_norenorm", 303, T=2, N=160, d=128, f=128, E=4, k=2, cf=1.5, dtype="bf16", flags=2),
    "bf16_e96_k3": Config("add_e96", 304, T=2, N=130, d=256, f=128, E=96, k=3, cf=2.0, dtype="bf16"),
    "bf16_wide": Config("add_wide", 305, T=1, N=70, d=1152, f=128, E=40, k=1, cf=1.0, dtype="bf16"),
    "bf16_e256_k8": Config("add_e256", 306, T=2, N=90, d=128, f=128, E=256, k=8, cf=2.0, dtype="bf16"),
    "bf16_e32": Config("add_e32", 307, T=3, N=131, d=256, f=128, E=32, k=2, cf=1.25, dtype="bf16", bias="drift"),
    "one_token": Config("add_one", 308, T=2, N=1, d=256, f=128, E=4, k=2, cf=1.0, dtype="bf16"),
}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__
    __graft_entry__.build()


@pytest.mark.parametrize("name", list(CASES))
def test_dlogits_add(name):
    cfg = CASES[name]
    inp = workloads.make_inputs(cfg)
    p = problem_of(cfg)
    r = vm.StepRunner(p, to_dev(inp))
    r.step()
    b, i = r.b, r.inp
    dx0 = b.dx.clone()
    g = torch.Generator().manual_seed(cfg.index)
    aux = torch.randn(cfg.T, cfg.N, cfg.E, generator=g)
    b.dlogits.copy_(aux)
    q = problem_of(cfg, cfg.flags | vm.VMOE_DLOGITS_ADD)
    vm.vmoe_router_bwd(q, i["x"], i["w_router"], b.logits, b.idx, b.gate, b.slot, i["dy"], b.ye, b.dgate, b.dlogits,
                       b.dw_router, b.dbias, b.dx)
    torch.cuda.synchronize()
    dgate, dl, _, _, _ = oracle.router_bwd(inp["x"], inp["w_router"], b.logits, b.idx.cpu(), b.gate, b.slot.cpu(),
                                           inp["dy"], b.ye, cfg.flags)
    x, w = np64(inp["x"]), np64(inp["w_router"])
    dl = np.asarray(dl).reshape(cfg.T, cfg.N, cfg.E) + np64(aux)
    xtol = F32_TOL if cfg.dtype == "f32" else BF16_TOL
    checks = {"dgate": (b.dgate, dgate, cfg.T, F32_TOL), "dlogits": (b.dlogits, dl, cfg.T, F32_TOL),
              "dw": (b.dw_router, np.einsum("tnd,tne->tde", x, dl), cfg.T, F32_TOL),
              "dbias": (b.dbias, dl.sum(axis=1), cfg.T, F32_TOL),
              "dx": (b.dx, np64(dx0) + np.einsum("tde,tne->tnd", w, dl), cfg.T * cfg.N, xtol)}
    for n, (got, ref, groups, tol) in checks.items():
        assert rel_err(got, ref, None, groups) <= tol, n


def test_step_with_balance_losses_is_the_sum_of_its_parts():
    """StepRunner(balance=...): its dlogits are the plain step's plus vmoe_balance_bwd's, one fp32 addition."""
    cfg = CASES["bf16_top2"]
    inp = to_dev(workloads.make_inputs(cfg))
    p = problem_of(cfg)
    plain = vm.StepRunner(p, inp, router_grad=True)
    plain.step()
    r = vm.StepRunner(p, inp, router_grad=True, balance=(0.1, 0.05, 0.01))
    r.step()
    d = torch.empty_like(r.b.dlogits)
    o = r.balance
    vm.vmoe_balance_bwd(p, r.b.logits, None, o.count, o.tokens, o.excess, o.dloss, d)
    torch.cuda.synchronize()
    assert torch.equal(r.b.dlogits, plain.b.dlogits + d) and torch.equal(r.b.dgate, plain.b.dgate)
    assert int(o.count.sum()) == cfg.T * cfg.N * cfg.k and torch.equal(r.b.y, plain.b.y)
    assert torch.equal(torch.minimum(o.count, torch.tensor(r.b.C, device="cuda")), r.b.load)


def test_balance_needs_the_router():
    cfg = CASES["bf16_top2"]
    with pytest.raises(ValueError):
        vm.StepRunner(problem_of(cfg), to_dev(workloads.make_inputs(cfg)), balance=(1, 0, 0))
    with pytest.raises(ValueError):
        vm.BalanceBuffers(problem_of(cfg), (1.0, 2.0))
