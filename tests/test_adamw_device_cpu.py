"""A table of AdamW's tensors is for the device that it was made on (CPU: the library is a stand-in)."""
import pytest
import torch

import paper_2608_16188_gb300 as vm


def test_another_current_device_is_refused(monkeypatch):
    """Its kernel would be launched there, on addresses of this one."""
    calls, current = [], [0]

    class Library:
        def vmoe_adamw(self, *a):
            calls.append(a[0])
            return vm.VMOE_OK

    monkeypatch.setattr(vm, "library", lambda: Library())
    monkeypatch.setattr(vm, "_device", lambda: current[0])
    monkeypatch.setattr(vm, "_stream", lambda s: 0)
    monkeypatch.setattr(vm, "_arrays", lambda where, *a: [None if t is None else t.data_ptr() for t, _, _ in a])
    z = lambda: torch.zeros(64)  # noqa: E731
    table = vm.adamw_tensors([dict(param=z(), grad=z(), m=z(), v=z())])
    vm.vmoe_adamw(table, 1, 1e-3)
    current[0] = 1
    with pytest.raises(vm.VmoeError) as e:
        vm.vmoe_adamw(table, 2, 1e-3)
    assert e.value.status == vm.VMOE_ERR_INVALID and calls == [1]
    vm.vmoe_adamw(vm.adamw_tensors([]), 1, 1e-3)  # nothing on any device
