"""VMOE_DLOGITS_ADD where nothing writes the gradients that are added to (CPU)."""
import pytest
import torch

import paper_2608_16188_gb300 as vm


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__
    __graft_entry__.build()


def test_the_flag_alone_is_refused_where_no_one_can_write_them():
    """Each step would add its gradients to those of the step before."""
    p = vm.problem(2, 4, 8, 8, 2, 1, 1.0, "f32", flags=vm.VMOE_DLOGITS_ADD)
    w = dict(w_router=torch.zeros(2, 8, 2), w1=torch.zeros(2, 2, 8, 8), w2=torch.zeros(2, 2, 8, 8))
    with pytest.raises(ValueError, match="DLOGITS_ADD"):
        vm.BlockStack(p, [w], device="cpu")
    with pytest.raises(ValueError, match="DLOGITS_ADD"):
        vm.HostPipeline(p, w, device="cpu")
    st = vm.BlockStack(p, [w], balance=(0.1, 0.0, 0.0), device="cpu")  # the losses' gradients are written first
    assert st.runners[0].p_add.flags == vm.VMOE_DLOGITS_ADD
    vm.StepRunner(p, dict(w, x=torch.zeros(2, 4, 8)), vm.Buffers(p, "cpu"), router_grad=True)  # the caller writes b.dlogits
