"""Refusals of vmoe_head_loss and vmoe_head_loss_bwd: argument checks run before any CUDA call."""
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


def _p(T=2, N=64, d=64, dtype="bf16"):
    return vm.problem(T, N, d, 8, 1, 1, 1.0, dtype)


FWD = ("z", "w", "label", "tidx", "tlogit", "ce", "lse", "kl", "tlse", "logp", "ws")
BWD = ("z", "w", "label", "tidx", "tlogit", "ce", "lse", "tlse", "logp", "dce", "dlse", "dkl", "dz", "dw", "ws")


def _call(fn, names, head, p=None, nbytes=1 << 40, **kw):
    a = dict.fromkeys(names, P)
    a.update(kw)
    return fn(ctypes.byref(p or _p()), ctypes.byref(head) if head else None, *a.values(), nbytes, None)


def test_head_refusals():
    lib, head = vm.library(), vm.head_config(100, 8, 2.0)
    for fn, names in ((lib.vmoe_head_loss, FWD), (lib.vmoe_head_loss_bwd, BWD)):
        call = lambda h=head, **kw: _call(fn, names, h, **kw)  # noqa: E731
        for n in names:
            assert call(**{n: P + 4}) == INVALID, n
        for n in ("z", "w", "label", "tidx", "tlogit", "ce", "lse", "tlse", "logp", "ws"):
            assert call(**{n: None}) == INVALID, n
        for h in (None, vm.head_config(0), vm.head_config(100, -1), vm.head_config(100, 8, 0.0), vm.head_config(100, 8, -1.0),
                  vm.head_config(100, 8, float("inf")), vm.head_config(100, 8, float("nan")), vm.head_config(100, 8, 1e-42),
                  vm.VmoeHead(100, 8, 1.0, 2)):
            assert call(h) == INVALID
        assert call(vm.head_config(100, 129)) == UNSUPPORTED and call(vm.head_config((1 << 20) + 1, 8)) == UNSUPPORTED
        assert call(p=_p(d=65544)) == UNSUPPORTED and call(vm.head_config((1 << 30) + 1)) == UNSUPPORTED
        assert call(vm.head_config(100)) == INVALID  # a teacher's arrays without a teacher
        assert call(p=_p(T=1, N=(1 << 25), d=8), h=vm.head_config(1 << 30, 8)) == UNSUPPORTED
        least = vm.vmoe_head_min_workspace_size(_p(), head)
        assert call(nbytes=least - 1) == INVALID and call(nbytes=0) == INVALID
        assert lib.vmoe_head_loss(None, ctypes.byref(head), *[P] * 11, 1 << 40, None) == INVALID
    none = dict(label=None, ce=None, lse=None)
    assert _call(lib.vmoe_head_loss_bwd, BWD, head, **none) == INVALID  # dce without a label
    assert _call(lib.vmoe_head_loss_bwd, BWD, head, dz=None, dw=None) == INVALID
    assert _call(lib.vmoe_head_loss_bwd, BWD, head, dce=None, dlse=None, dkl=None) == INVALID
    off = dict(tidx=None, tlogit=None, tlse=None, logp=None)
    assert _call(lib.vmoe_head_loss_bwd, BWD, vm.head_config(100), **off) == INVALID  # dkl without a teacher
    assert _call(lib.vmoe_head_loss, FWD, vm.head_config(100), kl=None, **none, **off) == INVALID  # neither


def test_workspace_sizes():
    for p in (_p(), _p(N=1), _p(dtype="f32")):
        for head in (vm.head_config(1), vm.head_config(50000), vm.head_config(50000, 32, 2.0, True)):
            least, most = vm.vmoe_head_min_workspace_size(p, head), vm.vmoe_head_workspace_size(p, head)
            assert 0 < least <= most
    assert vm.vmoe_head_workspace_size(_p(), vm.head_config(0)) == 0
    assert vm.vmoe_head_min_workspace_size(_p(d=12), vm.head_config(10)) == 0


def test_binding_refuses_other_tensors():
    p, head = _p(), vm.head_config(100)
    for z in (torch.zeros(2, 64, 64), torch.zeros(2, 64, 63, dtype=torch.bfloat16), torch.zeros(2, 64, 64, dtype=torch.bfloat16)):
        with pytest.raises(vm.VmoeError) as e:
            vm.vmoe_head_loss(p, head, z, P, P, None, None, P, P, None, None, None, P, 1 << 40)
        assert e.value.status == INVALID


def test_head_and_gate_buffers_refuse_what_does_not_fit():
    p = _p()
    w = torch.zeros(2, 100, 64, dtype=torch.bfloat16)
    for kw in (dict(labels=False), dict(w=torch.zeros(100, dtype=torch.bfloat16))):
        with pytest.raises(ValueError):
            vm.Head(p, **dict(dict(w=w, device="cpu"), **kw))
    head = vm.Head(p, w, device="cpu")
    with pytest.raises(RuntimeError):
        head.backward(torch.zeros(2, 64))
    assert not head.shared and vm.Head(p, w[0], device="cpu", train=False).parameters() == []
    for bias in (torch.zeros(2, 7), torch.zeros(2, 8, dtype=torch.float64), torch.zeros(8, 2).t()):
        with pytest.raises(ValueError):
            vm.GateBuffers(vm.problem(2, 64, 64, 8, 8, 2, 1.0), vm.gating(), bias, device="cpu")


def test_a_temperature_whose_factor_is_infinite():
    """log2(e) / temperature is what logits are taken times: past fp32's range a logit of 0 would be NaN."""
    lib, least = vm.library(), vm.vmoe_head_min_workspace_size(_p(), vm.head_config(100, 8, 4.5e-39))
    assert least > 0
    for head in (vm.head_config(100, 8, 4e-39), vm.head_config(100, 8, 1e-42)):
        assert vm.vmoe_head_min_workspace_size(_p(), head) == 0
        assert _call(lib.vmoe_head_loss, FWD, head) == INVALID and _call(lib.vmoe_head_loss_bwd, BWD, head) == INVALID
