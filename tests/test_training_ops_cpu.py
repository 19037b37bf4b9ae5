"""Refusals of the balance losses, block norms and AdamW: argument checks run before any CUDA call."""
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


def test_balance_refusals():
    lib = vm.library()
    p = vm.problem(2, 64, 8, 8, 4, 2, 1.0, "f32")
    ws = vm.vmoe_balance_workspace_size(p)
    assert ws > 0
    good = [P, P, None, P, P, P, P, P, ws]
    call = lambda a, q=p: lib.vmoe_balance(ctypes.byref(q), *a, None)  # noqa: E731
    for i in (0, 1, 3, 4, 5, 6, 7):
        for v in (None, P + 4):
            assert call(good[:i] + [v] + good[i + 1:]) == INVALID, (i, v)
    assert call(good[:2] + [P + 1] + good[3:]) == INVALID
    assert call(good[:8] + [ws - 1]) == INVALID
    assert lib.vmoe_balance(None, *good, None) == INVALID
    bad = vm.problem(2, 64, 8, 8, 4, 5, 1.0, "f32")
    assert call(good, bad) == INVALID and vm.vmoe_balance_workspace_size(bad) == 0
    assert call(good, vm.problem(2, 64, 8, 8, 300, 2, 1.0, "f32")) == UNSUPPORTED
    back = [P, None, P, P, P, P, P]
    for i in (0, 2, 3, 4, 5, 6):
        assert lib.vmoe_balance_bwd(ctypes.byref(p), *(back[:i] + [None] + back[i + 1:]), None) == INVALID


def test_block_norm_refusals():
    lib = vm.library()
    p = vm.problem(2, 64, 64, 8, 1, 1, 1.0, "bf16")
    cfg = vm.norm_config()

    def fwd(x=P, y=P, post_w=P, post_b=P, gate=P, pre_w=P, pre_b=P, z=P, u=P, ps=P, qs=P, cfg=cfg, p=p):
        return lib.vmoe_block_norm(ctypes.byref(p), ctypes.byref(cfg) if cfg else None, x, y, post_w, post_b, gate, pre_w, pre_b, z, u, ps, qs, None)

    none = dict(y=None, z=None, post_w=None, post_b=None, gate=None, ps=None)
    bad = [dict(x=None), dict(x=P + 8), dict(z=None), dict(y=None), dict(none, u=None, pre_w=None, pre_b=None, qs=None),
           dict(none, gate=P), dict(none, ps=P), dict(u=None), dict(u=None, pre_w=None, pre_b=None), dict(gate=P + 4),
           dict(cfg=vm.norm_config(post=False)), dict(cfg=vm.norm_config(eps=0.0)), dict(cfg=vm.norm_config(eps=float("nan"))),
           dict(cfg=vm.norm_config(residual_scale=float("inf"))), dict(cfg=vm.VmoeNorm(1e-6, 1.0, 4)), dict(cfg=None)]
    for kw in bad:
        assert fwd(**kw) == INVALID, kw
    assert fwd(p=vm.problem(2, 64, 8200, 8, 1, 1, 1.0, "bf16")) == UNSUPPORTED
    assert fwd(p=vm.problem(1024, 1 << 21, 8, 8, 1, 1, 1.0, "bf16")) == UNSUPPORTED
    assert vm.vmoe_block_norm_bwd_workspace_size(vm.problem(2, 64, 8200, 8, 1, 1, 1.0, "bf16")) == 0

    ws = vm.vmoe_block_norm_bwd_workspace_size(p)
    names = ("y", "z", "ps", "qs", "post_w", "post_b", "gate", "pre_w", "dz", "du", "dx", "dy", "dpost_w", "dpost_b", "dgate",
             "dpre_w", "dpre_b", "ws", "nbytes")

    def bwd(cfg=cfg, **kw):
        a = dict.fromkeys(names, P)
        a.update(nbytes=ws)
        a.update(kw)
        return lib.vmoe_block_norm_bwd(ctypes.byref(p), ctypes.byref(cfg), *(a[n] for n in names), None)

    branch = dict(y=None, dy=None, post_w=None, post_b=None, gate=None, dpost_w=None, dpost_b=None, dgate=None)
    no_u = dict(du=None, pre_w=None, dpre_w=None, dpre_b=None)
    for kw in (dict(dx=None), dict(dy=None), dict(y=None), dict(z=None), dict(ps=None), dict(qs=None), dict(du=None),
               dict(no_u, dz=None), dict(branch, **no_u), dict(branch, gate=P), dict(branch, dgate=P), dict(post_w=None),
               dict(gate=None), dict(pre_w=None), dict(nbytes=ws - 1), dict(ws=None), dict(dz=P + 2),
               dict(cfg=vm.norm_config(post=False))):
        assert bwd(**kw) == INVALID, kw


def _entry(**kw):
    e = vm.VmoeAdamwTensor(P, P, P, P, None, None, None, 100, vm.VMOE_BF16, vm.VMOE_BF16, vm.VMOE_STATE_F32, 1.0, 0.0)
    for k, v in kw.items():
        setattr(e, k, v)
    return e


def _adamw(entries, **kw):
    c = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, seed=0, step_dev=None, lr_dev=None, grad_scale=None)
    c.update(kw)
    table = (vm.VmoeAdamwTensor * max(1, len(entries)))(*entries)
    return vm.library().vmoe_adamw(len(entries), table, ctypes.byref(vm.VmoeAdamwConfig(*c.values())), None)


def test_adamw_refusals():
    nan, inf = float("nan"), float("inf")
    for kw in (dict(lr=nan), dict(lr=inf), dict(lr=1e39), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=nan), dict(eps=0.0),
               dict(eps=-1.0), dict(eps=1e-60), dict(step=0), dict(step=-1, step_dev=P), dict(step_dev=P + 2),
               dict(grad_scale=P + 1), dict(lr_dev=P + 3)):
        assert _adamw([_entry()], **kw) == INVALID, kw
    e4 = dict(state=vm.VMOE_STATE_E4M3, m_scale=P, v_scale=P)
    for kw in (dict(param=None), dict(grad=None), dict(m=None), dict(v=P + 4), dict(numel=-1), dict(param_dtype=2),
               dict(grad_dtype=-1), dict(state=2), dict(m_scale=P), dict(state=1), dict(e4, v_scale=None),
               dict(e4, m_scale=P + 2), dict(master=P + 8), dict(lr_scale=nan), dict(weight_decay=inf)):
        assert _adamw([_entry(), _entry(**kw)]) == INVALID, kw
    f32 = dict(param_dtype=vm.VMOE_F32)
    assert _adamw([_entry(**f32)]) == UNSUPPORTED  # fp32 parameters, bf16 gradients
    assert _adamw([_entry(**f32, grad_dtype=vm.VMOE_F32, master=P)]) == UNSUPPORTED
    assert _adamw([_entry(numel=1 << 38)]) == UNSUPPORTED
    lib = vm.library()
    assert lib.vmoe_adamw(-1, None, None, None) == INVALID and lib.vmoe_adamw(1, None, ctypes.byref(vm.VmoeAdamwConfig()), None) == INVALID
    # nothing to do, nothing launched: no GPU needed
    assert _adamw([]) == vm.VMOE_OK
    assert _adamw([_entry(numel=0, param=None, grad=None, m=None, v=None)]) == vm.VMOE_OK


def test_the_binding_refuses_tensors_it_would_misread():
    """Host tensors, another dtype, too few elements or a stride: a raw pointer of them would be read as another
    array, or past its end."""
    p = vm.problem(2, 4, 8, 8, 1, 1, 1.0, "f32")
    x = torch.zeros(2, 4, 8)
    with pytest.raises(vm.VmoeError) as e:
        vm.vmoe_block_norm(p, vm.norm_config(post=False), x, None, None, None, None, None, None, None, x)
    assert e.value.status == INVALID
    with pytest.raises(vm.VmoeError):
        vm.vmoe_balance_bwd(p, torch.zeros(2, 4, 1), None, P, P, P, P, P)
    with pytest.raises(vm.VmoeError):
        vm.adamw_tensors([dict(param=x, grad=x, m=x, v=x)])
    with pytest.raises(vm.VmoeError):
        vm.adamw_tensors([dict(param=x.half(), grad=x, m=x, v=x)])


def test_dlogits_add_is_a_known_flag():
    p = vm.problem(2, 64, 128, 256, 4, 2, 1.25, "bf16", flags=vm.VMOE_DLOGITS_ADD)
    assert vm.vmoe_problem_capacity(p) == 40


def test_a_stack_refuses_its_own_buffers_as_input():
    """The backward reads x again: an x that the forward or the backward overwrites gives another gradient."""
    p = vm.problem(2, 4, 8, 8, 2, 1, 1.0, "f32")
    w = dict(w_router=torch.zeros(2, 8, 2), w1=torch.zeros(2, 2, 8, 8), w2=torch.zeros(2, 2, 8, 8))
    st = vm.BlockStack(p, [w, w], device="cpu")
    for x in (st.z[0], st.z[-1], st.z[-1].view(-1), st.dz):
        with pytest.raises(ValueError, match="copy"):
            st.forward(x)
    assert st.x is None


def test_states_of_a_parameter_that_requires_a_gradient_hold_no_graph(monkeypatch):
    """The master copy of a leaf is plain memory: not a node of a graph that keeps the leaf's history."""
    import paper_2608_16188_gb300.optim as optim
    monkeypatch.setattr(optim, "adamw_tensors", lambda t: t)  # host tensors have no table
    w = torch.zeros(512, dtype=torch.bfloat16, requires_grad=True)
    o = vm.AdamW([dict(param=w, grad=torch.zeros_like(w))])
    assert not o.tensors[0]["master"].requires_grad
