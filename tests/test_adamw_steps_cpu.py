"""The step's number of AdamW (CPU: the call itself is replaced)."""
import pytest
import torch

import paper_2608_16188_gb300 as vm
import paper_2608_16188_gb300.optim as optim


@pytest.fixture()
def calls(monkeypatch):
    """The numbers t that vmoe_adamw was called for; it raises while the list `refuse` holds anything."""
    seen, refuse = [], []

    def call(table, step, *a, stream=None, **kw):
        if refuse:
            raise vm.VmoeError(vm.VMOE_ERR_INVALID, "vmoe_adamw")
        dev = a[5] if len(a) > 5 else None
        seen.append(step + (0 if dev is None else int(dev)))

    monkeypatch.setattr(optim, "adamw_tensors", lambda t: t)
    monkeypatch.setattr(optim, "vmoe_adamw", call)
    monkeypatch.setattr(optim, "_stream", lambda s: s)
    return seen, refuse


@pytest.mark.parametrize("capturable", [False, True])
def test_a_refused_step_is_not_counted(calls, capturable):
    seen, refuse = calls
    o = vm.AdamW([dict(param=torch.zeros(8), grad=torch.zeros(8))], capturable=capturable)
    o.step()
    refuse.append(True)
    for _ in range(3):
        with pytest.raises(vm.VmoeError):
            o.step(grad_scale=torch.ones(2))
    refuse.clear()
    o.step()
    assert seen == [1, 2] and o.steps == 2
    assert not capturable or int(o.step_dev) == 2
