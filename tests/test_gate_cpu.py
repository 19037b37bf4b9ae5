"""Refusals of vmoe_gate, vmoe_gate_bwd and vmoe_gate_bias: argument checks run before any CUDA call."""
import ctypes

import pytest
import torch

import paper_2608_16188_gb300 as vm

P = 1 << 20  # an aligned, never dereferenced address
INVALID, UNSUPPORTED = vm.VMOE_ERR_INVALID, vm.VMOE_ERR_UNSUPPORTED


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__
    __graft_entry__.build()


def _p(**kw):
    a = dict(T=2, N=64, d=64, f=8, E=8, k=2, cf=1.25, dtype="bf16", flags=0)
    a.update(kw)
    return vm.problem(*a.values())


def test_gate_refusals():
    lib = vm.library()
    ws = vm.vmoe_gate_workspace_size(_p())
    assert ws > 0
    names = ("x", "w", "lb", "sb", "mask", "logits", "idx", "gate", "slot", "load", "demand", "ws", "nbytes")

    def call(p=None, cfg=vm.gating("sigmoid", 4, 2, 2, 2.5), **kw):
        a = dict.fromkeys(names, P)
        a.update(nbytes=ws)
        a.update(kw)
        return lib.vmoe_gate(ctypes.byref(p or _p()), ctypes.byref(cfg) if cfg else None, *a.values(), None)

    for n in ("x", "w", "logits", "idx", "gate", "slot", "load", "ws"):
        assert call(**{n: None}) == INVALID, n
    for n in names[:-1]:
        assert call(**{n: P + 4}) == INVALID, n
    assert call(nbytes=ws - 1) == INVALID
    given = _p(flags=vm.VMOE_LOGITS_IN)
    assert call(given, logits=None, x=None, w=None) == INVALID
    for cfg in (None, vm.gating(2), vm.gating(-1), vm.gating(groups=0), vm.gating(groups=3), vm.gating(groups=4, groups_kept=0),
                vm.gating(groups=4, groups_kept=5), vm.gating(groups=8, groups_kept=1), vm.gating(groups=8, groups_kept=2, group_top=2),
                vm.gating(group_top=0), vm.gating(group_top=3), vm.gating(scale=0.0), vm.gating(scale=-1.0),
                vm.gating(scale=float("inf")), vm.gating(scale=float("nan"))):
        assert call(cfg=cfg) == INVALID, cfg and [getattr(cfg, f) for f, _ in cfg._fields_]
    assert call(_p(k=9)) == INVALID and call(_p(E=300)) == UNSUPPORTED
    assert vm.vmoe_gate_workspace_size(_p(k=9)) == 0
    big = vm.problem(64, 1 << 25, 8, 8, 8, 2, 1.0)
    assert call(big, nbytes=1 << 60) == UNSUPPORTED


def test_gate_bwd_refusals():
    lib = vm.library()
    names = ("x", "w", "logits", "idx", "gate", "slot", "dy", "ye", "dgate", "dlogits", "dw", "dbias", "dx_in", "dx")

    def call(cfg=vm.gating(), **kw):
        a = dict.fromkeys(names, P)
        a.update(kw)
        return lib.vmoe_gate_bwd(ctypes.byref(_p()), ctypes.byref(cfg), *a.values(), None)

    for n in ("x", "logits", "idx", "gate", "slot", "dy", "ye", "dgate", "dlogits", "dw"):
        assert call(**{n: None}) == INVALID, n
    assert call(dx_in=None) == INVALID and call(dx=None) == INVALID and call(w=None) == INVALID
    assert call(cfg=vm.gating(groups=3)) == INVALID
    assert lib.vmoe_gate_bias(ctypes.byref(_p()), None, 0.1, P, None) == INVALID
    assert lib.vmoe_gate_bias(ctypes.byref(_p()), P, 0.1, None, None) == INVALID
    assert lib.vmoe_gate_bias(ctypes.byref(_p()), P, float("nan"), P, None) == INVALID


def test_binding_refuses_other_tensors():
    """A wrong size, dtype or order, and host memory, before the library is called."""
    p = _p(flags=vm.VMOE_LOGITS_IN)
    for logits in (torch.zeros(2, 64, 7), torch.zeros(2, 64, 8, dtype=torch.float64), torch.zeros(2, 8, 64).transpose(1, 2),
                   torch.zeros(2, 64, 8)):
        with pytest.raises(vm.VmoeError) as e:
            vm.vmoe_gate(p, vm.gating(), None, None, None, P, None, logits, P, P, P, P, P, P, 1 << 20)
        assert e.value.status == INVALID or logits.is_contiguous()
