"""Blocks as they are trained: norms, expert layers, balance losses and AdamW in one run.

The reference is autograd in 64 bits over the same blocks, with the routing (chosen experts, slots) that the
GPU took.  fp32 problems: each stage is held to 1e-5 of its output's RMS (or of the element) elsewhere; a
gradient passes at most 8 stages a block each way, two blocks: 32 x 1e-5 = 3.2e-4.
"""
import pytest
import torch

import paper_2608_16188_gb300 as vm
from gpu_helpers import rel_err

pytestmark = pytest.mark.gpu

TOL = 3.2e-4
WEIGHTS = (0.3, 0.2, 0.05)


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__
    __graft_entry__.build()


def _layers(T, N, d, f, E, L, dtype, rms, post, seed=0):
    g = torch.Generator().manual_seed(seed)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    out = []
    for _ in range(L):
        w = dict(w_router=r(T, d, E) / d ** 0.5, bias=0.3 * r(T, E), w1=(r(T, E, d, f) / d ** 0.5).to(dt),
                 w2=(r(T, E, f, d) / f ** 0.5).to(dt), pre_w=1 + 0.1 * r(T, d), gate=0.5 + 0.1 * r(T, d))
        if not rms:
            w["pre_b"] = 0.1 * r(T, d)
        if post:
            w["post_w"] = 1 + 0.1 * r(T, d)
            if not rms:
                w["post_b"] = 0.1 * r(T, d)
        out.append({k: v.cuda() for k, v in w.items()})
    x, dz = r(T, N, d).to(dt).cuda(), r(T, N, d).to(dt).cuda()
    return out, x, dz


def _norm64(v, w, b, rms, eps):
    if not rms:
        v = v - v.mean(dim=2, keepdim=True)
    v = v / torch.sqrt((v * v).mean(dim=2, keepdim=True) + eps)
    v = v * w[:, None, :]
    return v if b is None else v + b[:, None, :]


def _reference(st, layers, x, dz, rms, post, rho, eps, mask):
    """Gradients of <dz, z> + the weighted balance losses by autograd, fp64, routing from the GPU."""
    T, N, d = x.shape
    leaves = [{k: v.detach().double().cpu().requires_grad_() for k, v in w.items()} for w in layers]
    x64 = x.detach().double().cpu().requires_grad_()
    z, total = x64, 0.0
    on = torch.ones(T, N, dtype=torch.double) if mask is None else (mask.cpu() != 0).double()
    for w, r in zip(leaves, st.runners):
        idx, slot = r.b.idx.cpu().long(), r.b.slot.cpu()
        E, k = w["w_router"].shape[2], idx.shape[2]
        u = _norm64(z, w["pre_w"], w.get("pre_b"), rms, eps)
        logits = torch.einsum("tnd,tde->tne", u, w["w_router"]) + w["bias"][:, None, :]
        gates = torch.softmax(torch.gather(logits, 2, idx), dim=2) * (slot >= 0)
        per = torch.zeros(T, N, E, dtype=torch.double).scatter_add(2, idx, gates)
        h = torch.einsum("tnd,tedf->tenf", u, w["w1"])
        a = 0.5 * h * (1 + torch.erf(h / 2 ** 0.5))
        y = torch.einsum("tenf,tefd,tne->tnd", a, w["w2"], per)
        b = _norm64(y, w["post_w"], w.get("post_b"), rms, eps) if post else y
        z = rho * z + w["gate"][:, None, :] * b
        m = on.sum(dim=1)
        p = torch.softmax(logits, dim=2) * on[:, :, None]
        count = torch.zeros(T, E, dtype=torch.double)
        for t in range(T):
            count[t] = torch.bincount(idx[t][on[t] > 0].reshape(-1), minlength=E).double()
        imp = p.sum(dim=1)
        l0 = E / (k * m * m) * (count * imp).sum(dim=1)
        l1 = E / (m * m) * ((imp - m[:, None] / E) ** 2).sum(dim=1)
        l2 = (torch.logsumexp(logits, dim=2) ** 2 * on).sum(dim=1) / m
        total = total + (WEIGHTS[0] * l0 + WEIGHTS[1] * l1 + WEIGHTS[2] * l2).sum()
    (total + (z * dz.double().cpu()).sum()).backward()
    return z.detach(), x64.grad, [{k: v.grad for k, v in w.items()} for w in leaves]


@pytest.mark.parametrize("rms,post,masked", [(False, True, False), (True, True, True), (False, False, True)])
def test_gradients_of_a_stack(rms, post, masked):
    T, N, d, f, E, k, L, rho, eps = 2, 60, 64, 128, 4, 2, 2, 1.1, 1e-5
    layers, x, dz = _layers(T, N, d, f, E, L, "f32", rms, post, seed=1 + rms)
    p = vm.problem(T, N, d, f, E, k, 1.0, "f32")
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
    bad = {}
    for n, got, ref in [("z", z, rz), ("dx", dx, rdx)]:
        bad[n] = rel_err(got, ref)
    for i, (g, ref) in enumerate(zip(st.grads, rg)):
        for n, v in g.items():
            if v is not None:
                bad["%d.%s" % (i, n)] = rel_err(v, ref[n])
    assert len(bad) == 2 + sum(v is not None for g in st.grads for v in g.values())
    bad = {n: v for n, v in bad.items() if not v <= TOL}
    assert not bad, bad


@pytest.mark.parametrize("dtype,eight", [("f32", False), ("bf16", True)])
def test_training_steps_replayed_from_a_graph(dtype, eight):
    """Forward, backward and update captured once and replayed agree bitwise with eager steps, and the update
    is AdamW's of the stack's own gradients."""
    T, N, d, f, E, k, L = 2, 96, 128, 256, 4, 2, 2
    p = vm.problem(T, N, d, f, E, k, 1.25, dtype)

    def make():
        layers, x, dz = _layers(T, N, d, f, E, L, dtype, False, True, seed=9)
        st = vm.BlockStack(p, layers, balance=WEIGHTS)
        opt = vm.AdamW(st.parameters(), lr=1e-3, eight_bit=eight, capturable=True, seed=4)
        return layers, x, dz, st, opt

    def step(x, dz, st, opt):
        st.forward(x)
        st.backward(dz)
        opt.step()

    la, xa, dza, sa, oa = make()
    lb, xb, dzb, sb, ob = make()
    assert len(oa.tensors) == L * 9
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(xa, dza, sa, oa)
    start = {n: v.clone() for n, v in lb[0].items()}
    for i in range(3):
        graph.replay()
        step(xb, dzb, sb, ob)
        torch.cuda.synchronize()
        for wa, wb in zip(la, lb):
            for n in wa:
                assert torch.equal(wa[n], wb[n]), (i, n)
    assert int(oa.step_dev) == 3 and vm.vmoe_device_status() == 0
    for n, v in lb[0].items():  # every parameter moved by its rate, no further than three times that
        t = [t for t in ob.tensors if t["param"] is v][0]
        moved = (t.get("master", v).float() - start[n].float()).abs()
        assert float(moved.max()) > 0 and float(moved.max()) < 3.2e-3 + (0.02 if v.dtype == torch.bfloat16 else 0.0), n


def test_another_stream_gives_the_same():
    T, N, d, f, E, k, L = 2, 50, 128, 128, 4, 1, 1
    p = vm.problem(T, N, d, f, E, k, 1.25, "bf16")
    out = []
    for stream in (None, torch.cuda.Stream()):
        layers, x, dz = _layers(T, N, d, f, E, L, "bf16", True, False, seed=3)
        st = vm.BlockStack(p, layers, vm.norm_config(rms=True, post=False), balance=WEIGHTS)
        opt = vm.AdamW(st.parameters(), eight_bit=True, capturable=True)
        torch.cuda.synchronize()
        st.forward(x, stream)
        dx = st.backward(dz, stream)
        opt.step(stream=stream)
        torch.cuda.synchronize()
        out.append([dx] + [t["param"] for t in opt.tensors] + [t["m"].float() for t in opt.tensors])
    assert all(torch.equal(a, b) for a, b in zip(*out))


def test_misuse_is_refused():
    layers, x, dz = _layers(1, 8, 128, 128, 2, 1, "bf16", False, True)
    p = vm.problem(1, 8, 128, 128, 2, 1, 1.0, "bf16")
    with pytest.raises(ValueError):
        vm.BlockStack(p, [])
    st = vm.BlockStack(p, layers)
    with pytest.raises(RuntimeError):
        st.backward(dz)
    with pytest.raises(vm.VmoeError):
        st.forward(x.float())
    with pytest.raises(vm.VmoeError):  # a strided gradient
        w = layers[0]["w1"]
        vm.AdamW([dict(param=w, grad=w.transpose(-1, -2))])
    with pytest.raises(vm.VmoeError):  # the same tensor twice: a race
        g = torch.zeros_like(layers[0]["w1"])
        vm.AdamW([dict(param=layers[0]["w1"], grad=g), dict(param=layers[0]["w1"], grad=g)])
