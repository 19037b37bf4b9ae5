"""bf16 blocks as they are trained: gradients and updates against references, on a GB300.

Gradients against autograd in 64 bits with the GPU's routing.  Each stage's output is held to 5e-3 of its RMS
(the aggregate bar of the parity tests); a gradient passes at most 8 stages a block each way, two blocks.  Roundings
of 32 stages are independent: sqrt(32) x 5e-3 = 2.8e-2, and three times that for the stages that
amplify what they get (a norm's 1 / deviation, the differences in a softmax's backward): 9e-2 of the RMS.

Updates against AdamW in 64 bits from the stack's own gradients, on the fp32 master copy: 4e-6 of the update and two
roundings, 2^-23, of the parameter.  The weights themselves are the master copy's nearest.
"""
import numpy as np
import pytest
import torch

import paper_2608_16188_gb300 as vm
from gpu_helpers import np64, rms_err
from oracle import training as tr
from test_gpu_block_stack import WEIGHTS, _layers, _reference

pytestmark = pytest.mark.gpu

TOL = 9e-2


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__
    __graft_entry__.build()


@pytest.mark.parametrize("rms,post,masked", [(False, True, False), (True, True, True), (False, False, True)])
def test_gradients_of_a_bf16_stack(rms, post, masked):
    T, N, d, f, E, k, L, rho, eps = 2, 60, 128, 256, 4, 2, 2, 1.1, 1e-5
    layers, x, dz = _layers(T, N, d, f, E, L, "bf16", rms, post, seed=21 + rms)
    p = vm.problem(T, N, d, f, E, k, 1.0, "bf16")
    mask = None
    if masked:
        mask = torch.ones(T, N, dtype=torch.uint8, device="cuda")
        mask[0, 40:] = 0
    st = vm.BlockStack(p, layers, vm.norm_config(rms=rms, post=post, eps=eps, residual_scale=rho), balance=WEIGHTS, token_mask=mask)
    z = st.forward(x)
    dx = st.backward(dz)
    torch.cuda.synchronize()
    assert vm.vmoe_device_status() == 0
    rz, rdx, rg = _reference(st, layers, x, dz, rms, post, rho, eps, mask)
    err = {"z": rms_err(z, rz), "dx": rms_err(dx, rdx)}
    for i, (g, ref) in enumerate(zip(st.grads, rg)):
        err.update({"%d.%s" % (i, n): rms_err(v, ref[n]) for n, v in g.items() if v is not None})
    assert len(err) == 2 + sum(v is not None for g in st.grads for v in g.values())
    assert all(v <= TOL for v in err.values()), err


@pytest.mark.parametrize("eight", [False, True])
def test_updates_of_a_bf16_stack(eight):
    """The first step (moments of zero are exact in 8 bits too): every parameter of every block."""
    T, N, d, f, E, k, L = 2, 96, 128, 256, 4, 2, 2
    p = vm.problem(T, N, d, f, E, k, 1.25, "bf16")
    layers, x, dz = _layers(T, N, d, f, E, L, "bf16", False, True, seed=9)
    st = vm.BlockStack(p, layers, balance=WEIGHTS)
    opt = vm.AdamW(st.parameters(), lr=1e-3, weight_decay=0.05, eight_bit=eight, seed=4)
    before = [np64(t["param"]).reshape(-1) for t in opt.tensors]
    st.forward(x)
    st.backward(dz)
    opt.step()
    torch.cuda.synchronize()
    assert len(opt.tensors) == L * 9
    moved = 0
    for t, b in zip(opt.tensors, before):
        new, _, _, upd = tr.adamw(b, np64(t["grad"]).reshape(-1), 0.0, 0.0, 1, 1e-3, 0.9, 0.999, 1e-8, weight_decay=t["weight_decay"])
        got = t.get("master", t["param"])
        assert np.all(np.abs(np64(got).reshape(-1) - new) <= 2.0 ** -23 * np.abs(b) + 4e-6 * upd + 1e-12)
        moved += int((np.abs(new - b) > 5e-4).sum())
        if "master" in t:
            assert t["param"].dtype == torch.bfloat16 and torch.equal(t["param"], t["master"].to(torch.bfloat16))
    assert moved > 0.5 * sum(b.size for b in before)  # what does not move shows
