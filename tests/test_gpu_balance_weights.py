"""Weights of the balance losses that change between steps and between replays of a captured one, on a GB300."""
import pytest
import torch

import paper_2608_16188_gb300 as vm
import workloads
from gpu_helpers import problem_of, to_dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__
    __graft_entry__.build()


def test_weights_changed_in_place_reach_the_gradient():
    """A step whose weights were changed in place, eager and replayed, agrees bitwise with one made with them."""
    cfg = workloads.Config("weights", 401, T=2, N=60, d=128, f=128, E=4, k=2, cf=1.25, dtype="bf16", bias="drift")
    inp, p = to_dev(workloads.make_inputs(cfg)), problem_of(cfg)
    w = torch.zeros(cfg.T, 3, device="cuda")
    r = vm.StepRunner(p, inp, router_grad=True, balance=w)
    r.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r.step()
    for i, values in enumerate(([[0.5, 0.0, 0.0], [0.0, 0.1, 0.2]], [[0.1, 0.2, 0.3], [3.0, 0.0, 0.0]])):
        w.copy_(torch.tensor(values))
        other = vm.StepRunner(p, inp, router_grad=True, balance=torch.tensor(values, device="cuda"))
        other.step()
        r.step() if i == 0 else graph.replay()
        torch.cuda.synchronize()
        for n in ("dlogits", "dw_router", "dbias", "dx"):
            assert torch.equal(getattr(r.b, n), getattr(other.b, n)), (i, n)
    plain = vm.StepRunner(p, inp, router_grad=True)
    plain.step()
    assert not torch.equal(plain.b.dlogits, r.b.dlogits)
