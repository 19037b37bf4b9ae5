"""Offsets past 31 and 32 bits: tensors of more than 2^31 elements (2^32 for AdamW) against small ones that they
repeat, on a GB300.  Tolerances as in the operators' own tests; sums of repeats are summed in other runs: 1e-5."""
import numpy as np
import pytest
import torch

import paper_2608_16188_gb300 as vm
from gpu_helpers import np64
from oracle import training as tr

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__
    __graft_entry__.build()


@pytest.fixture(autouse=True)
def _free():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("eight", [False, True])
def test_adamw_past_2_to_32_elements(eight):
    """Only the last 1000 elements and the first 256 have gradients; the others stay what they were."""
    n, tail = (1 << 32) + 1000, 1000
    new = lambda dt, k=n: torch.zeros(k, dtype=dt, device="cuda")  # noqa: E731
    p, g = new(torch.bfloat16), new(torch.bfloat16)
    gen = torch.Generator().manual_seed(3)
    ends = torch.cat([torch.arange(256), torch.arange(n - tail, n)])
    p[ends.cuda()] = torch.randn(256 + tail, generator=gen).to(torch.bfloat16).cuda()
    g[ends.cuda()] = torch.randn(256 + tail, generator=gen).to(torch.bfloat16).cuda()
    kind = torch.float8_e4m3fn if eight else torch.float32
    t = dict(param=p, grad=g, m=new(kind), v=new(kind))
    if eight:
        t.update(m_scale=new(torch.float32, (n + 255) // 256), v_scale=new(torch.float32, (n + 255) // 256))
    before = np64(p[-tail:])
    vm.vmoe_adamw(vm.adamw_tensors([t]), 1, 1e-2, seed=9)
    torch.cuda.synchronize()
    rp, rm, rv, upd = tr.adamw(before, np64(g[-tail:]), 0.0, 0.0, 1, 1e-2, 0.9, 0.999, 1e-8)
    got = np64(p[-tail:])
    assert np.all(np.abs(got - rp) <= 2.0 ** -8 * np.abs(rp) + 4e-6 * upd + 2.0 ** -23 * np.abs(before))
    assert int((p[256:n - tail] != 0).sum()) == 0 and int((p[:256] != 0).sum()) > 200
    if not eight:
        assert np.all(np.abs(np64(t["m"][-tail:]) - rm) <= 2.0 ** -22 * np.abs(rm) + 1e-30)
        return
    first = n - tail - (n - tail) % 256  # whole blocks from here on
    lead = n - tail - first
    bits = tr.dither_bits(n - first, 0, 1, 9, first)
    for k, val, b in (("m", rm, bits[0]), ("v", np.sqrt(rv), bits[1])):
        q, scale, border, _ = tr.e4m3_encode(np.concatenate([np.zeros(lead), val]), b)
        far = border > 2e-4
        assert np.array_equal(np64(t[k][first:])[far], q[far])
        assert np.allclose(np64(t[k + "_scale"][first // 256:]), scale, rtol=2.0 ** -21, atol=0)


def test_balance_past_2_to_31_logits():
    T, tile, reps, E, k = 2, 1024, 4400, 256, 4
    N = tile * reps
    assert T * N * E > 1 << 31
    g = torch.Generator().manual_seed(5)
    x = torch.randn(T, tile, E, generator=g).cuda()
    idx = x.topk(k, dim=2).indices.to(torch.int32)
    dl = torch.rand(T, 3, generator=g).cuda()

    def run(x, idx):
        p = vm.problem(T, x.shape[1], 8, 8, E, k, 1.0, "f32")
        o = dict(count=torch.empty(T, E, dtype=torch.int32, device="cuda"), tokens=torch.empty(T, dtype=torch.int32, device="cuda"),
                 excess=torch.empty(T, E, device="cuda"), loss=torch.empty(T, 3, device="cuda"), dlogits=torch.empty_like(x))
        ws = torch.empty(vm.vmoe_balance_workspace_size(p), dtype=torch.uint8, device="cuda")
        vm.vmoe_balance(p, x, idx, None, o["count"], o["tokens"], o["excess"], o["loss"], ws)
        vm.vmoe_balance_bwd(p, x, None, o["count"], o["tokens"], o["excess"], dl, o["dlogits"])
        torch.cuda.synchronize()
        return o

    a, b = run(x, idx), run(x.repeat(1, reps, 1), idx.repeat(1, reps, 1))
    assert torch.equal(b["count"], a["count"] * reps) and b["tokens"].tolist() == [N] * T
    scale = float(a["excess"].abs().max())
    assert float((b["excess"] / reps - a["excess"]).abs().max()) <= 1e-5 * scale
    assert torch.allclose(a["loss"], b["loss"], rtol=2e-5, atol=0)
    top = float(a["dlogits"].abs().max())
    for at in (0, reps // 2, reps - 1):  # a gradient of a mean: 1 / reps of the tile's
        part = b["dlogits"][:, at * tile:(at + 1) * tile] * reps
        assert float((part - a["dlogits"]).abs().max()) <= 2e-5 * top


def test_block_norm_past_2_to_31_elements():
    T, tile, reps, d = 3, 512, 1400, 1024
    N = tile * reps
    assert T * N * d > 1 << 31
    g = torch.Generator().manual_seed(7)
    r = lambda *s: torch.randn(*s, generator=g).cuda()  # noqa: E731
    s = {n: r(T, tile, d).to(torch.bfloat16) for n in ("x", "y", "dz", "du")}
    par = [1 + 0.1 * r(T, d), 0.1 * r(T, d), 0.5 + 0.1 * r(T, d), 1 + 0.1 * r(T, d), 0.1 * r(T, d)]

    def run(s):
        p, cfg = vm.problem(T, s["x"].shape[1], d, 8, 1, 1, 1.0, "bf16"), vm.norm_config()
        like = lambda: torch.empty_like(s["x"])  # noqa: E731
        z, u, dx, dy = like(), like(), like(), like()
        ps, qs = (torch.empty(T, s["x"].shape[1], 2, device="cuda") for _ in range(2))
        grads = [torch.empty(T, d, device="cuda") for _ in range(5)]
        ws = torch.empty(vm.vmoe_block_norm_bwd_workspace_size(p), dtype=torch.uint8, device="cuda")
        vm.vmoe_block_norm(p, cfg, s["x"], s["y"], *par, z, u, ps, qs)
        vm.vmoe_block_norm_bwd(p, cfg, s["y"], z, ps, qs, par[0], par[1], par[2], par[3], s["dz"], s["du"], dx, dy, *grads, ws)
        torch.cuda.synchronize()
        return dict(z=z, u=u, dx=dx, dy=dy), grads

    (a, ga), (b, gb) = run(s), run({n: v.repeat(1, reps, 1) for n, v in s.items()})
    for n in a:
        for at in (0, reps // 2, reps - 1):
            assert torch.equal(b[n][:, at * tile:(at + 1) * tile], a[n]), n
    for x, y in zip(ga, gb):
        assert float((y / reps - x).abs().max()) <= 1e-5 * float(x.abs().max())
