"""What BlockStack refuses as input or gradient because its own calls overwrite it (CPU: nothing is launched)."""
import pytest
import torch

import paper_2608_16188_gb300 as vm
import paper_2608_16188_gb300.block as block


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__
    __graft_entry__.build()


def _stack(balance=None, layers=2):
    p = vm.problem(2, 4, 8, 8, 2, 1, 1.0, "f32")
    w = dict(w_router=torch.zeros(2, 8, 2), w1=torch.zeros(2, 2, 8, 8), w2=torch.zeros(2, 2, 8, 8), pre_w=torch.ones(2, 8))
    return vm.BlockStack(p, [dict(w) for _ in range(layers)], balance=balance, device="cpu")


@pytest.mark.parametrize("balance", [None, (0.1, 0.1, 0.1)])
def test_an_input_in_any_buffer_of_the_stack_is_refused(balance):
    """The backward reads x again: one that the forward or the backward overwrites gives another gradient."""
    st = _stack(balance)
    own = [*st.z, st.dz, st.workspace]
    for r in st.runners:
        own += [r.inp["x"], r.inp["dy"], r.b.y, r.b.dx, r.b.xe, r.b.h, r.b.dw1, r.b.logits]
        own += [] if balance is None else [r.balance.excess]
    for g in st.grads:
        own += [v for v in g.values() if v is not None]
    for t in own:
        for x in (t, t.view(-1), t.view(-1)[-1:], t.view(-1)[:1]):
            with pytest.raises(ValueError, match="copy"):
                st.forward(x)
    assert st.x is None


def test_other_tensors_are_taken(monkeypatch):
    """Not a buffer, also where it lies right beside one."""
    seen = []
    monkeypatch.setattr(block, "_stream", lambda s: None)
    monkeypatch.setattr(block, "vmoe_block_norm", lambda *a: seen.append(a[2]))
    st = _stack()
    monkeypatch.setattr(vm.StepRunner, "forward", lambda self, stream=None: None)
    for x in (torch.zeros(2, 4, 8), st.layers[0]["w1"], torch.zeros(1 << 16)[:64].view(2, 4, 8)):
        st.forward(x)
        assert st.x is x
    begin = st._own[0][0]
    assert all(b[1] <= a[0] for a, b in zip(st._own[1:], st._own)) and begin > 0  # bisection needs them apart


def test_a_gradient_in_a_buffer_that_is_written_meanwhile_is_refused(monkeypatch):
    monkeypatch.setattr(block, "_stream", lambda s: None)
    for n in ("vmoe_block_norm", "vmoe_block_norm_bwd"):
        monkeypatch.setattr(block, n, lambda *a, **k: None)
    for n in ("forward", "backward"):
        monkeypatch.setattr(vm.StepRunner, n, lambda self, stream=None: None)
    st = _stack()
    st.forward(torch.zeros(2, 4, 8))
    for dz in (st.runners[-1].inp["dy"], st.runners[-1].inp["dy"].view(-1)[8:], st.dz.view(-1)[8:]):
        with pytest.raises(ValueError, match="copy"):
            st.backward(dz)
    for dz in (st.z[-1], st.dz, torch.zeros(2, 4, 8)):
        assert st.backward(dz) is st.dz
