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


def _opt(sizes, **kw):
    return vm.AdamW([dict(param=torch.randn(n).to(torch.bfloat16), grad=torch.zeros(n, dtype=torch.bfloat16)) for n in sizes], **kw)


@pytest.mark.parametrize("capturable", [False, True])
def test_a_state_is_taken_over_in_place(calls, capturable):
    seen, _ = calls
    a, b = (_opt((300, 5000), eight_bit=True, seed=s, capturable=c) for s, c in ((7, not capturable), (1, capturable)))
    for _ in range(3):
        a.step()
    for t in a.tensors:
        for k in a.STATE:
            if t.get(k) is not None:
                t[k].copy_(torch.rand(t[k].shape))
    kept = [{k: t.get(k) for k in b.STATE} for t in b.tensors]
    b.load_state_dict(a.state_dict())
    assert b.seed == 7 and [sorted(s) for s in a.state_dict()["tensors"]] == [["m", "master", "v"], ["m", "m_scale", "master", "v", "v_scale"]]
    for t, s, k in zip(a.tensors, b.tensors, kept):
        for n in b.STATE:
            assert s.get(n) is k[n]  # the addresses that the table holds
            assert k[n] is None or torch.equal(k[n].view(torch.uint8), t[n].view(torch.uint8)), n
    seen.clear()
    b.step()
    assert seen == [4] and b.state_dict()["step"] == 4


def test_a_state_of_something_else_is_refused(calls):
    o = _opt((300, 5000), eight_bit=True)
    before = [t["m"].clone() for t in o.tensors]
    for other in (_opt((300,), eight_bit=True), _opt((300, 5001), eight_bit=True), _opt((300, 5000)),
                  _opt((300, 5000), eight_bit=True, master=False)):
        for t in other.tensors:
            t["m"].fill_(1.0)
        with pytest.raises(ValueError):
            o.load_state_dict(other.state_dict())
    assert all(torch.equal(t["m"].view(torch.uint8), m.view(torch.uint8)) for t, m in zip(o.tensors, before)) and o.steps == 0


def test_master_copies_follow_parameters_that_were_loaded(calls):
    o = _opt((300, 20))
    for t in o.tensors:
        t["param"].fill_(2.5)
    o.refresh_master()
    assert all(torch.all(t["master"] == 2.5) for t in o.tensors)
