"""The balance losses' weights are the caller's tensor, or refused (CPU: nothing is launched)."""
import pytest
import torch

import paper_2608_16188_gb300 as vm


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__
    __graft_entry__.build()


def test_a_tensor_of_weights_is_kept_and_a_strided_one_refused():
    """A strided tensor would have to be copied, and what the caller writes into it later would be lost."""
    p = vm.problem(4, 8, 8, 8, 2, 1, 1.0, "f32")
    w = torch.rand(4, 3)
    b = vm.BalanceBuffers(p, w, device="cpu")
    w[2, 1] = 7.0
    assert float(b.dloss[2, 1]) == 7.0
    for bad in (torch.rand(1, 3).expand(4, 3), torch.rand(3, 4).t(), torch.rand(4, 6)[:, ::2], torch.rand(4, 3).double(), torch.rand(3)):
        with pytest.raises(ValueError, match="contiguous"):
            vm.BalanceBuffers(p, bad, device="cpu")
    three = vm.BalanceBuffers(p, (0.5, 0.25, 0.125), device="cpu")
    assert three.dloss.tolist() == [[0.5, 0.25, 0.125]] * 4
