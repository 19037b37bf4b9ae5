"""A negative count of workspace bytes is refused before the library reads it as a huge one (CPU)."""
import pytest

import paper_2608_16188_gb300 as vm

P = 1 << 20  # an aligned, never dereferenced address


@pytest.fixture(autouse=True)
def _lib(monkeypatch):
    import __graft_entry__
    __graft_entry__.build()

    class Refusing:  # stands for the library: a call that reaches it would launch
        def __getattr__(self, name):
            def call(*a):
                if name == "vmoe_status_string":
                    return b"status"
                raise AssertionError("%s was called" % name)
            return call

    monkeypatch.setattr(vm, "library", lambda: Refusing())


def test_negative_counts_do_not_reach_the_library():
    p, norm = vm.problem(2, 64, 128, 128, 4, 2, 1.0, "bf16"), vm.norm_config()
    for n in (-1, -(1 << 40)):
        for call in (lambda: vm.vmoe_balance(p, *[P] * 7, P, n, stream=0),
                     lambda: vm.vmoe_block_norm_bwd(p, norm, *[P] * 17, P, n, stream=0),
                     lambda: vm.vmoe_expert_bwd(p, *[P] * 10, P, n, stream=0),
                     lambda: vm.vmoe_attn_expert_bwd(p, 2, *[P] * 11, P, n, stream=0)):
            with pytest.raises(vm.VmoeError) as e:
                call()
            assert e.value.status == vm.VMOE_ERR_INVALID
