"""HostPipeline with balance losses: every step's losses, counts and padding are its own, on a GB300."""
import pytest
import torch

import paper_2608_16188_gb300 as vm
import workloads
from gpu_helpers import problem_of, to_dev

pytestmark = pytest.mark.gpu

WEIGHTS = (0.3, 0.2, 0.05)


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__
    __graft_entry__.build()


def _setup(steps, seed=3):
    cfg = workloads.Config("pipe_balance", 402, T=3, N=197, d=256, f=512, E=4, k=2, cf=1.25, dtype="bf16", bias="drift")
    inp, p = to_dev(workloads.make_inputs(cfg)), problem_of(cfg)
    g = torch.Generator().manual_seed(seed)
    pin = lambda t: t.pin_memory()  # noqa: E731
    r = lambda: pin(torch.randn(inp["x"].shape, generator=g).to(torch.bfloat16))  # noqa: E731
    mask = lambda: pin((torch.arange(cfg.N) < torch.randint(1, cfg.N + 1, (cfg.T, 1), generator=g)).to(torch.uint8))  # noqa: E731
    ins = [(r(), r(), mask()) for _ in range(steps)]
    empty = lambda *s, dt=torch.float32: pin(torch.full(s, -7, dtype=dt))  # noqa: E731
    outs = [(torch.empty_like(ins[0][0]).pin_memory(), torch.empty_like(ins[0][0]).pin_memory(), empty(cfg.T, 3),
             empty(cfg.T, cfg.E, dt=torch.int32)) for _ in range(steps)]
    return cfg, p, inp, ins, outs


def _reference(p, inp, x, dy, mask):
    i = dict(inp, x=x.cuda(), dy=dy.cuda(), token_mask=None if mask is None else mask.cuda())
    r = vm.StepRunner(p, i, router_grad=True, balance=WEIGHTS)
    r.step()
    torch.cuda.synchronize()
    return r


def test_losses_counts_and_padding_of_every_step():
    cfg, p, inp, ins, outs = _setup(5)
    ins[2] = ins[2][:2]            # no mask: the one of the weights
    ins[3] = (*ins[3][:2], None)
    outs[1] = outs[1][:3]          # the losses alone
    outs[4] = (*outs[4][:2], None, outs[4][3])
    fixed = torch.ones(cfg.T, cfg.N, dtype=torch.uint8)
    fixed[:, 50:] = 0
    weights = dict({k: v for k, v in inp.items() if k not in ("x", "dy")}, token_mask=fixed.cuda())
    pipe = vm.HostPipeline(p, weights, router_grad=True, balance=WEIGHTS)
    for _ in range(2):  # twice: the second run starts in the first one's slots
        pipe.run(ins, outs)
    torch.cuda.synchronize()
    last = None
    for i, (a, o) in enumerate(zip(ins, outs)):
        mask = a[2] if len(a) > 2 and a[2] is not None else fixed
        last = _reference(p, inp, a[0], a[1], mask)
        assert torch.equal(o[0], last.b.y.cpu()) and torch.equal(o[1], last.b.dx.cpu()), i
        if o[2] is not None:
            assert torch.equal(o[2], last.balance.loss.cpu()), i
        if len(o) > 3:
            assert torch.equal(o[3], last.balance.count.cpu()), i
    assert torch.equal(pipe.slots[0].balance.loss, last.balance.loss)
    assert torch.equal(pipe.slots[0].b.dw_router, last.b.dw_router)
    assert vm.vmoe_device_status() == 0


def test_without_extra_entries_the_steps_are_the_same():
    cfg, p, inp, ins, outs = _setup(3, seed=8)
    weights = {k: v for k, v in inp.items() if k not in ("x", "dy")}
    pipe = vm.HostPipeline(p, weights, router_grad=True, balance=WEIGHTS)
    pipe.run([a[:2] for a in ins], [o[:2] for o in outs])
    torch.cuda.synchronize()
    for a, o in zip(ins, outs):
        r = _reference(p, inp, a[0], a[1], None)
        assert torch.equal(o[0], r.b.y.cpu()) and torch.equal(o[1], r.b.dx.cpu())


def test_what_the_losses_need_is_refused_without_them():
    cfg, p, inp, ins, outs = _setup(1)
    weights = {k: v for k, v in inp.items() if k not in ("x", "dy")}
    plain = vm.HostPipeline(p, weights)
    for i, o in ((ins, [outs[0][:2]]), ([ins[0][:2]], outs)):
        with pytest.raises(ValueError, match="balance"):
            plain.run(i, o)
    pipe = vm.HostPipeline(p, weights, router_grad=True, balance=WEIGHTS)
    for bad in (ins[0][2].bool(), ins[0][2][:1], ins[0][2].float()):
        with pytest.raises(ValueError, match="mask"):
            pipe.run([(*ins[0][:2], bad)], [outs[0][:2]])
