"""Offsets past 31 and 32 bits in heads and gates, on a GB300: weights, gradients by the logits, logits of routers.

Large runs against small ones on the entries or tokens that matter.  Losses of the two differ by their sums' roundings (1e-5
of the loss); a bf16 gradient by a whole step, 2^-7 of its value, where its sum falls to either side of a border, and by dl's
own roundings, 2^-8 of the terms, where the terms are not the same numbers.
"""
import pytest
import torch

import paper_2608_16188_gb300 as vm

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__
    __graft_entry__.build()


@pytest.fixture(autouse=True)
def _free():
    yield
    torch.cuda.empty_cache()


def _run(p, head, z, w, label, dce, nbytes=None):
    o = dict(ce=torch.empty(p.T, p.N, device="cuda"), lse=torch.empty(p.T, p.N, device="cuda"))
    ws = torch.empty(nbytes or vm.vmoe_head_workspace_size(p, head), dtype=torch.uint8, device="cuda")
    vm.vmoe_head_loss(p, head, z, w, label, None, None, o["ce"], o["lse"], None, None, None, ws)
    o.update(dz=torch.full_like(z, float("nan")), dw=torch.full_like(w, float("nan")))
    vm.vmoe_head_loss_bwd(p, head, z, w, label, None, None, o["ce"], o["lse"], None, None, dce, None, None, o["dz"], o["dw"], ws)
    return o


@pytest.mark.parametrize("N", [3, 40])
def test_weights_past_2_to_32_elements(N):
    """Only the first and the last 500 of 2^22 + 1001 entries have weights; the others' logits are 0."""
    V, d, E = (1 << 22) + 1001, 1024, 500
    g = torch.Generator().manual_seed(N)
    ends = (torch.randn(2 * E, d, generator=g) / 8).to(torch.bfloat16).cuda()
    w = torch.zeros(V, d, dtype=torch.bfloat16, device="cuda")
    w[:E], w[V - E:] = ends[:E], ends[E:]
    z = torch.randn(1, N, d, generator=g).to(torch.bfloat16).cuda()
    label = torch.randint(V - E, V, (1, N), generator=g).to(torch.int32).cuda()
    label[0, 0] = 1
    dce = torch.rand(1, N, generator=g).cuda()
    p, head = vm.problem(1, N, d, 8, 1, 1, 1.0), vm.head_config(V, shared=True)
    o = _run(p, head, z, w, label, dce)
    torch.cuda.synchronize()
    assert vm.vmoe_device_status() == 0
    zd, wd = z[0].double(), ends.double()
    l = zd @ wd.t()
    top = l.amax(1, keepdim=True).clamp(min=0)
    lse = top[:, 0] + torch.log(torch.exp(l - top).sum(1) + (V - 2 * E) * torch.exp(-top[:, 0]))
    at = torch.where(label[0].long() < E, label[0].long(), label[0].long() - V + 2 * E)
    assert float((o["lse"][0] - lse).abs().max()) <= 1e-5 * float(lse.abs().max())
    assert float((o["ce"][0] - (lse - l.gather(1, at[:, None])[:, 0])).abs().max()) <= 1e-5 * float(lse.abs().max())
    dl = torch.exp(l - lse[:, None]) * dce[0].double()[:, None]
    dl[torch.arange(N), at] -= dce[0].double()
    for got, want, size in ((o["dz"][0], dl @ wd, dl.abs() @ wd.abs()),
                            (torch.cat([o["dw"][:E], o["dw"][V - E:]]), dl.t() @ zd, dl.abs().t() @ zd.abs())):
        assert bool(((got.double() - want).abs() <= 2.0 ** -7 * size + 1e-30).all())
    rest = torch.exp(-lse) * dce[0].double() @ zd  # an entry's gradient where its logits are 0
    for v in (E, V // 2, V - E - 1):
        size = torch.exp(-lse) * dce[0].double() @ zd.abs()
        assert bool(((o["dw"][v].double() - rest).abs() <= 2.0 ** -7 * size + 1e-30).all())


def test_gradients_by_the_logits_past_2_to_32_elements():
    """66000 tokens by 65536 entries in one piece, 4.3e9 of them, and in many."""
    N, V, d = 66000, 65536, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    z = torch.randn(1, N, d, generator=g, device="cuda").to(torch.bfloat16)
    w = (torch.randn(V, d, generator=g, device="cuda") / 4).to(torch.bfloat16)
    label = torch.randint(0, V, (1, N), generator=g, device="cuda").to(torch.int32)
    dce = torch.rand(1, N, generator=g, device="cuda")
    p, head = vm.problem(1, N, d, 8, 1, 1, 1.0), vm.head_config(V, shared=True)
    need = vm.vmoe_head_workspace_size(p, head)
    one, many = _run(p, head, z, w, label, dce, need + (10 << 30)), _run(p, head, z, w, label, dce)
    few = slice(N - 100, N)
    last = _run(vm.problem(1, 100, d, 8, 1, 1, 1.0), head, *(t[:, few].contiguous() if t.dim() > 1 and t.shape[1] == N else t
                                                             for t in (z, w, label, dce)))
    assert vm.vmoe_device_status() == 0
    assert torch.equal(one["ce"], many["ce"]) and float((one["ce"][:, few] - last["ce"]).abs().max()) <= 1e-5 * float(one["ce"].max())
    # the call of 100 tokens keeps dl to 2^-16, the others round it to bf16: up to 2^-8 of each term of dz, 2^-8 sum |dl| |w|
    # together, beside the two outputs' roundings, 2^-8 |dz| each
    zf, wf = z[0, few].float(), w.float()
    dl = torch.exp(zf @ wf.t() - one["lse"][0, few, None])
    dl[torch.arange(100), label[0, few].long()] -= 1.0
    rounding = 2.0 ** -8 * ((dce[0, few, None] * dl).abs() @ wf.abs()).double()[None]
    for a, b, more in ((one["dz"], many["dz"], 0.0), (one["dw"], many["dw"], 0.0), (one["dz"][:, few], last["dz"], rounding)):
        a, b = a.double(), b.double()
        assert bool(((a - b).abs() <= 2.0 ** -7 * a.abs() + 2e-5 * a.abs().amax() + more).all())


def test_router_logits_past_2_to_31():
    """2^23 + 77 tokens over 256 experts: the last tokens' choices are those of a small call, and all are counted."""
    N, E, k = (1 << 23) + 77, 256, 4
    g = torch.Generator(device="cuda").manual_seed(2)
    logits = torch.randn(1, N, E, generator=g, device="cuda")
    bias = 0.1 * torch.randn(1, E, generator=g, device="cuda")
    cfg = vm.gating("sigmoid", 8, 4, 2)

    def run(l):
        n = l.shape[1]
        p = vm.problem(1, n, 8, 8, E, k, 1.0, "f32", vm.VMOE_LOGITS_IN)
        i32 = lambda *s: torch.full(s, -7, dtype=torch.int32, device="cuda")  # noqa: E731
        o = dict(idx=i32(1, n, k), gate=torch.empty(1, n, k, device="cuda"), slot=i32(1, n, k), load=i32(1, E), demand=i32(1, E))
        ws = torch.empty(vm.vmoe_gate_workspace_size(p), dtype=torch.uint8, device="cuda")
        vm.vmoe_gate(p, cfg, None, None, None, bias, None, l, o["idx"], o["gate"], o["slot"], o["load"], o["demand"], ws)
        return p, o
    p, o = run(logits)
    _, small = run(logits[:, -1000:].contiguous())
    assert torch.equal(o["idx"][:, -1000:], small["idx"]) and torch.equal(o["gate"][:, -1000:], small["gate"])
    count = torch.bincount(o["idx"].reshape(-1).long(), minlength=E)
    assert torch.equal(count, o["demand"][0].long())
    C = vm.vmoe_problem_capacity(p)
    assert torch.equal(o["load"][0].long(), count.clamp(max=C))
    # every kept place is taken once: slots of an expert are 0 to load - 1
    kept = o["slot"] >= 0
    place = o["idx"][kept].long() * C + o["slot"][kept].long()
    assert int(kept.sum()) == int(o["load"].sum()) and place.unique().numel() == place.numel()
    assert int(o["slot"].max()) == int(o["load"].max()) - 1
