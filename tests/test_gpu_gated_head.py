"""A training step from tokens to weights: blocks whose experts vmoe_gate chooses, a head with labels and a teacher,
AdamW and the gates' bias, in one run.

The reference is autograd in 64 bits over the same step, with the choices and slots that the GPU took.  fp32: each
stage is held to 1e-5 of its output's RMS (or of the element); a gradient passes at most 8 stages a block each way, two
blocks, and the head's two: 34 x 1e-5 = 3.4e-4.
"""
import pytest
import torch

import paper_2608_16188_gb300 as vm
import workloads
from gpu_helpers import problem_of, rel_err, to_dev
from oracle import gating

pytestmark = pytest.mark.gpu

TOL = 3.4e-4
TAU, SCALE = 2.0, 1.6


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__
    __graft_entry__.build()


def _setup(T, N, d, f, E, V, K, dtype, shared, seed=0):
    g = torch.Generator().manual_seed(seed)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    layers = []
    for _ in range(2):
        w = dict(w_router=r(T, d, E) / d ** 0.5, bias=0.3 * r(T, E), w1=(r(T, E, d, f) / d ** 0.5).to(dt),
                 w2=(r(T, E, f, d) / f ** 0.5).to(dt), pre_w=1 + 0.1 * r(T, d), gate=0.5 + 0.1 * r(T, d), post_w=1 + 0.1 * r(T, d))
        layers.append({k: v.cuda() for k, v in w.items()})
    w = (r(*((V, d) if shared else (T, V, d))) / d ** 0.5).to(dt).cuda()
    mask = torch.ones(T, N, dtype=torch.uint8)
    mask[0, N - N // 3:] = 0
    label = torch.randint(0, V, (T, N), generator=g)
    label[torch.rand(T, N, generator=g) < 0.3] = -100
    tidx = torch.randint(0, V, (T, N, K), generator=g)
    tidx[torch.rand(T, N, generator=g) < 0.3] = -1
    label[mask == 0], tidx[mask == 0] = -1, -1
    teach = dict(label=label.to(torch.int32).cuda(), teacher_idx=tidx.to(torch.int32).cuda(), teacher_logit=2 * r(T, N, K).cuda())
    up = [r(T, N).abs().cuda() / N for _ in range(2)]
    return layers, w, r(T, N, d).to(dt).cuda(), mask.cuda(), teach, up


def _norm(v, w):
    v = v / torch.sqrt((v * v).mean(dim=2, keepdim=True) + 1e-6)
    return v * w[:, None, :]


def _reference(st, layers, w, x, teach, up):
    T, N, d = x.shape
    leaves = [{k: v.detach().double().cpu().requires_grad_() for k, v in p.items()} for p in layers]
    w64, x64 = (t.detach().double().cpu().requires_grad_() for t in (w, x))
    z = x64
    for p, r in zip(leaves, st.runners):
        idx, slot = r.b.idx.cpu().long(), r.b.slot.cpu()
        E = p["w_router"].shape[2]
        u = _norm(z, p["pre_w"])
        logits = torch.einsum("tnd,tde->tne", u, p["w_router"]) + p["bias"][:, None, :]
        s = torch.sigmoid(logits.gather(2, idx.clamp(min=0))) * (idx >= 0)
        gates = SCALE * s / s.sum(dim=2, keepdim=True).clamp(min=1e-30) * (slot >= 0)
        per = torch.zeros(T, N, E, dtype=torch.double).scatter_add(2, idx.clamp(min=0), gates)
        h = torch.einsum("tnd,tedf->tenf", u, p["w1"])
        y = torch.einsum("tenf,tefd,tne->tnd", 0.5 * h * (1 + torch.erf(h / 2 ** 0.5)), p["w2"], per)
        z = z + p["gate"][:, None, :] * _norm(y, p["post_w"])
    l = z @ (w64.t() if w64.dim() == 2 else w64.transpose(1, 2))
    y, i, t = teach["label"].cpu().long(), teach["teacher_idx"].cpu().long(), teach["teacher_logit"].cpu().double()
    has, on = y >= 0, i >= 0
    ce = -torch.log_softmax(l, 2).gather(2, y.clamp(min=0)[..., None])[..., 0] * has
    logq = torch.log_softmax((t / TAU).masked_fill(~on, -1e300), 2)
    q = torch.exp(logq) * on
    kl = (q * (logq.masked_fill(~on, 0.0) - torch.log_softmax(l / TAU, 2).gather(2, i.clamp(min=0)))).sum(2) * on.any(2)
    ((up[0].cpu() * ce).sum() + (up[1].cpu() * kl).sum()).backward()
    return leaves, w64, x64, ce.detach(), kl.detach()


def _step(st, head, x, teach, up):
    head.forward(st.forward(x), **teach)
    return st.backward(head.backward(up[0], up[1]))


@pytest.mark.parametrize("shared", [False, True])
def test_gradients_of_a_training_step(shared):
    T, N, d, f, E, k, V, K = 2, 50, 64, 128, 8, 2, 300, 6
    layers, w, x, mask, teach, up = _setup(T, N, d, f, E, V, K, "f32", shared)
    p = vm.problem(T, N, d, f, E, k, 1.0, "f32")
    cfg = vm.gating("sigmoid", 4, 2, 2, SCALE)
    st = vm.BlockStack(p, layers, norm=vm.norm_config(rms=True), token_mask=mask, gating=cfg)
    for gate in st.gates:
        gate.select_bias.copy_(0.1 * torch.randn(T, E))
    head = vm.Head(p, w, teacher_k=K, temperature=TAU)
    dx = _step(st, head, x, teach, up)
    torch.cuda.synchronize()
    assert vm.vmoe_device_status() == 0
    for r in st.runners:  # the choices are those of the logits
        ref = gating.choose(r.b.logits.cpu(), r.gating.select_bias.cpu(), mask, k, r.b.C, "sigmoid", 4, 2, 2, True, SCALE)
        assert (r.b.idx.cpu().numpy() == ref["idx"]).all() and (r.b.slot.cpu().numpy() == ref["slot"]).all()
        assert (r.gating.demand.cpu().numpy() == ref["demand"]).all()
    leaves, w64, x64, ce, kl = _reference(st, layers, w, x, teach, up)
    assert rel_err(head.ce, ce.numpy()) <= TOL and rel_err(head.kl, kl.numpy()) <= TOL
    assert rel_err(head.dw, w64.grad.numpy()) <= TOL and rel_err(dx, x64.grad.numpy()) <= TOL
    for leaf, g in zip(leaves, st.grads):
        for name, v in leaf.items():
            assert rel_err(g[name], v.grad.numpy()) <= TOL, name


def test_steps_update_everything_and_replay():
    """bf16 steps with AdamW and the gates' bias, run and then captured: the replayed step is the same step."""
    T, N, d, f, E, k, V, K = 2, 197, 128, 256, 8, 2, 1000, 8
    layers, w, x, mask, teach, up = _setup(T, N, d, f, E, V, K, "bf16", True, seed=5)
    p = vm.problem(T, N, d, f, E, k, 1.25, "bf16")
    st = vm.BlockStack(p, layers, norm=vm.norm_config(rms=True), token_mask=mask, gating=vm.gating("sigmoid", 2, 1, 2, SCALE),
                       balance=(0.01, 0.0, 0.001))
    head = vm.Head(p, w, teacher_k=K, temperature=TAU)
    opt = vm.AdamW(st.parameters() + head.parameters(), lr=1e-3, capturable=True)
    keep = [t["param"].clone() for t in opt.tensors] + [t["master"].clone() for t in opt.tensors if "master" in t]

    def step():
        dx = _step(st, head, x, teach, up)
        opt.step()
        st.update_gates(0.01)
        return dx

    def reset():
        live = [t["param"] for t in opt.tensors] + [t["master"] for t in opt.tensors if "master" in t]
        for a, b in zip(live, keep):
            a.copy_(b)
        for t in opt.tensors:
            t["m"].zero_(), t["v"].zero_()
        for gate in st.gates:
            gate.select_bias.zero_()
        opt.step_dev.zero_()

    def run(n, go):
        reset()
        for _ in range(n):
            go()
        torch.cuda.synchronize()
        return [t["param"].clone() for t in opt.tensors] + [g.select_bias.clone() for g in st.gates] + [head.ce.clone(), head.kl.clone()]

    first = run(3, step)
    assert all(torch.isfinite(t.float()).all() for t in first)
    assert all(not torch.equal(a, b) for a, b in zip(first, keep[:len(opt.tensors)]))
    assert all((g.select_bias != 0).any() for g in st.gates)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step()
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.synchronize()
    again = run(3, graph.replay)
    assert vm.vmoe_device_status() == 0
    for a, b in zip(first, again):
        assert torch.equal(a, b)


def test_a_head_in_pieces_and_a_frozen_one():
    T, N, d, V = 2, 100, 128, 3000
    _, w, x, _, teach, up = _setup(T, N, d, 8, 1, V, 4, "bf16", False, seed=2)
    p = vm.problem(T, N, d, 8, 1, 1, 1.0, "bf16")
    whole = vm.Head(p, w, teacher_k=4, temperature=TAU)
    small = vm.Head(p, w, teacher_k=4, temperature=TAU, train=False,
                    workspace_bytes=vm.vmoe_head_min_workspace_size(p, whole.config))
    out = []
    for h in (whole, small):
        h.forward(x, **teach)
        out.append(h.backward(up[0], up[1]).clone())
    assert small.parameters() == [] and len(whole.parameters()) == 1
    assert torch.equal(whole.ce, small.ce) and torch.equal(whole.kl, small.kl)
    # the sums over the pieces are rounded apart: 12 roundings to fp32, which may take the two values to either side of a
    # border of bf16; each is then off by half a step, 2^-8 of itself, and the two by a whole one
    assert rel_err(out[1], out[0].double().cpu().numpy()) <= 2.0 ** -7 + 1e-5


def test_host_pipeline_with_gating():
    """Steps from pinned host memory, each with a mask of its own, choose as the step by itself does."""
    cfg = workloads.Config("pipe_gate", 403, T=3, N=197, d=256, f=512, E=4, k=2, cf=1.25, dtype="bf16", bias="drift")
    inp, p = to_dev(workloads.make_inputs(cfg)), problem_of(cfg)
    g = torch.Generator().manual_seed(3)
    r = lambda: torch.randn(inp["x"].shape, generator=g).to(torch.bfloat16).pin_memory()  # noqa: E731
    mask = lambda: (torch.arange(cfg.N) < torch.randint(1, cfg.N + 1, (cfg.T, 1), generator=g)).to(torch.uint8).pin_memory()  # noqa: E731
    ins = [(r(), r(), mask()), (r(), r()), (r(), r(), mask())]
    outs = [(torch.empty_like(ins[0][0]).pin_memory(), torch.empty_like(ins[0][0]).pin_memory()) for _ in ins]
    weights = {k: v for k, v in inp.items() if k not in ("x", "dy")}
    gate = vm.gating("sigmoid", 2, 1, 1)
    pipe = vm.HostPipeline(p, weights, router_grad=True, gating=gate)
    pipe.run(ins, outs)
    torch.cuda.synchronize()
    for a, o in zip(ins, outs):
        i = dict(inp, x=a[0].cuda(), dy=a[1].cuda(), token_mask=a[2].cuda() if len(a) > 2 else None)
        ref = vm.StepRunner(p, i, router_grad=True, gating=gate)
        ref.step()
        torch.cuda.synchronize()
        assert torch.equal(o[0], ref.b.y.cpu()) and torch.equal(o[1], ref.b.dx.cpu())
