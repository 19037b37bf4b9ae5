"""vmoe_head_loss and vmoe_head_loss_bwd against the fp64 oracle, on a GB300.

Tolerances, derived.  A logit is a sum of d products on tensor cores: bf16 products are exact in fp32 and each step of 16
is cut to fp32, off by at most one step of what has been summed: D = (d / 16 + 4) 2^-23 sum |z w|; fp32 operands take six
such sums and leave out products of parts below 3 * 2^-24 of |z w|: D = (6 d / 16 + 8) 2^-23 sum |z w|.  A dot product of
the teacher's entries is d / 32 fused steps a lane and a tree: below D.
lse moves by the largest D and the sum of exponentials (ex2.approx 2^-22, the sum's and logarithm's roundings): 1e-6
more, and its own rounding, 2^-23 of it.  ce and logp take twice that; kl their sum over q, and the teacher's own 4e-6.
dl: e^(l - lse) is off by 2 D + 4e-6 (|lse| + 1) 2^-2 relative to each of its terms (`size`), then rounded: 2^-8 of it in
bf16 (the parts of fp32 hold 2^-23).  dz and dw: that through the sums, sum |dl error| |w|, the sums' own steps (K / 16 + 8)
2^-23 sum |dl| |w|, and the output's rounding.
"""
import numpy as np
import pytest
import torch

import paper_2608_16188_gb300 as vm
from gpu_helpers import np64
from oracle import head as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__
    __graft_entry__.build()


def _inputs(T, N, V, d, K, dtype, shared, label, ragged, seed=0):
    g = torch.Generator().manual_seed(seed)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    z = torch.randn(T, N, d, generator=g)
    w = 1.5 / d ** 0.5 * torch.randn(*((V, d) if shared else (T, V, d)), generator=g)
    s = dict(label=None, tidx=None, tlogit=None)
    keep = torch.rand(T, N, generator=g) < (0.6 if ragged else 1.1)
    if label:
        y = torch.randint(0, V, (T, N), generator=g)
        for t in range(T):  # tokens that are sure of their answer among them
            z[t] += 8 * torch.rand(N, 1, generator=g) ** 3 * (w if shared else w[t])[y[t]]
        s["label"] = torch.where(keep, y, torch.randint(-5, 0, (T, N), generator=g)).to(torch.int32)
        if ragged and N > 3:
            s["label"][0, 2] = V  # outside
    if K:
        i = torch.randint(0, V, (T, N, K), generator=g)  # twice the same, now and then
        if label:
            i[..., 0] = y
        q = 3 * torch.randn(T, N, K, generator=g)
        if ragged:
            i[torch.rand(T, N, K, generator=g) < 0.2] = -1
            q[torch.rand(T, N, K, generator=g) < 0.1] = float("-inf")
            i[~keep] = -1
            if label:
                i[torch.rand(T, N, generator=g) < 0.3] = V + 3  # labels without a teacher
        s["tidx"], s["tlogit"] = i.to(torch.int32), q
    up = lambda: torch.randn(T, N, generator=g) / N  # noqa: E731
    s.update(dce=up() if label else None, dlse=0.1 * up() if label else None, dkl=up() if K else None)
    z, w = z.to(dt), w.to(dt)
    r = ref.loss(z, w, s["label"], s["tidx"], s["tlogit"], 1.0)
    z[torch.from_numpy(~(r["has"] | r["taught"]))] = float("nan")
    return z, w, s


def _dev(t):
    return None if t is None else t.cuda()


def _run(p, head, z, w, s, nbytes=None, stream=None, train=True, dz=True):
    T, N, K = p.T, p.N, head.teacher_k
    nan = lambda have, *sh: torch.full(sh, float("nan"), device="cuda") if have else None  # noqa: E731
    lab, tea = s["label"] is not None, K > 0
    o = dict(ce=nan(lab, T, N), lse=nan(lab, T, N), kl=nan(tea, T, N), tlse=nan(tea, T, N), logp=nan(tea, T, N, K))
    nbytes = vm.vmoe_head_workspace_size(p, head) if nbytes is None else nbytes
    ws = torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")
    zd, wd, y, i, q = z.cuda(), w.cuda(), _dev(s["label"]), _dev(s["tidx"]), _dev(s["tlogit"])
    vm.vmoe_head_loss(p, head, zd, wd, y, i, q, o["ce"], o["lse"], o["kl"], o["tlse"], o["logp"], ws, stream=stream)
    ws.fill_(255)
    o.update(dz=torch.full_like(zd, float("nan")) if dz else None, dw=torch.full_like(wd, float("nan")) if train else None)
    vm.vmoe_head_loss_bwd(p, head, zd, wd, y, i, q, o["ce"], o["lse"], o["tlse"], o["logp"], _dev(s["dce"]), _dev(s["dlse"]),
                          _dev(s["dkl"]), o["dz"], o["dw"], ws, stream=stream)
    return o


def _check(o, z, w, s, tau, dtype, few=False, flushed=0.0):
    r = ref.loss(z, w, s["label"], s["tidx"], s["tlogit"], tau)
    part = r["has"] | r["taught"]
    T, N, V = r["logits"].shape
    d = z.shape[2]
    za, wa = np.abs(np.where(part[..., None], np64(z), 0.0)), np.abs(np64(w))
    wt = np.broadcast_to(wa, (T,) + wa.shape) if wa.ndim == 2 else wa
    f32 = dtype == "f32"
    D = ((6 * d / 16 + 8) if f32 else (d / 16 + 4)) * 2.0 ** -23 * np.einsum("tnd,tvd->tnv", za, wt).max(axis=2)
    out = 2.0 ** -24 if f32 else 2.0 ** -8
    size_err = 2 * D
    for name, tem in (("lse", 1.0), ("tlse", tau)):
        if o.get(name) is None:
            continue
        tol = D / tem + 1e-6 + 2.0 ** -23 * np.abs(r[name])
        assert np.all(np.abs(np64(o[name]) - r[name]) <= np.where(r["has" if name == "lse" else "taught"], tol, 0)), name
        size_err = np.maximum(size_err, 2 * D / tem + 1e-6 * (np.abs(r[name]) + 1) + 3e-6)
    if o.get("ce") is not None:
        assert np.all(np.abs(np64(o["ce"]) - r["ce"]) <= np.where(r["has"], 2 * D + 2e-6 + 2.0 ** -22 * np.abs(r["ce"]), 0))
    if o.get("kl") is not None:
        tol = 2 * D / tau + 2e-6 + 2.0 ** -23 * np.abs(r["tlse"])
        lp = tol[..., None] + 2.0 ** -22 * np.abs(r["logp"])
        assert np.all(np.abs(np64(o["logp"]) - r["logp"]) <= np.where(r["taught"][..., None], lp, 0))
        qt = (r["q"] * (lp + 4e-6 * (1 + np.abs(r["logp"]) + np.abs(np.log(np.maximum(r["q"], 1e-30)))))).sum(axis=2)
        assert np.all(np.abs(np64(o["kl"]) - r["kl"]) <= qt + 2e-6 * r["taught"])
    dl, size = ref.dlogits(r, s["label"], s["tidx"], tau, s["dce"], s["dlse"], s["dkl"])
    dz, dw = ref.back(dl, z, w, part)
    err = size_err[..., None] * size + (2.0 ** -23 if f32 else 2.0 ** -16 if few else 2.0 ** -8) * np.abs(dl) + flushed
    steps = 6 if f32 else 1
    if o.get("dz") is not None:
        got = np64(o["dz"])
        tol = np.einsum("tnv,tvd->tnd", err + (steps * V / 16 + 8) * 2.0 ** -23 * np.abs(dl), wt) * (1 + out) + out * np.abs(dz)
        assert np.all(np.abs(got - dz) <= tol + 1e-38)
        assert np.all(got[~part] == 0)
    if o.get("dw") is not None:
        e = np.einsum("tnv,tnd->tvd", err + (steps * N * T / 16 + 8) * 2.0 ** -23 * np.abs(dl), za)
        e = e.sum(axis=0) if wa.ndim == 2 else e
        assert np.all(np.abs(np64(o["dw"]) - dw) <= e * (1 + out) + out * np.abs(dw) + 1e-38)
    return r


# (T, N, V, d): one token, one entry, ends inside and at a tile, odd sizes, widths from 8 on, more row tiles than a group
SIZES = [(1, 1, 1, 8), (1, 1, 1000, 384), (2, 3, 2, 64), (1, 256, 256, 64), (3, 257, 255, 72), (1, 197, 1000, 384),
         (2, 300, 2057, 200), (17, 20, 300, 128), (1, 700, 129, 768), (3, 16, 700, 72), (2, 17, 131, 64)]
MODES = {"ce": (True, 0, 1.0), "kd": (False, 9, 2.0), "both": (True, 33, 4.0), "both_tau1": (True, 5, 1.0), "kd_cold": (False, 128, 0.5)}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mode", list(MODES))
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_head_parity(size, mode, dtype):
    T, N, V, d = size
    label, K, tau = MODES[mode]
    shared = (T + N) % 2 == 0
    for ragged in ((False, True) if dtype == "bf16" else (True,)):
        z, w, s = _inputs(T, N, V, d, K, dtype, shared, label, ragged, seed=sum(size))
        p, head = vm.problem(T, N, d, 8, 1, 1, 1.0, dtype), vm.head_config(V, K, tau, shared)
        _check(_run(p, head, z, w, s), z, w, s, tau, dtype)
        assert vm.vmoe_device_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pieces_of_the_vocabulary(dtype):
    """The smallest workspace takes a tile of the vocabulary at a time; what is in between, some of them."""
    T, N, V, d, K = 2, 300, 1500, 136, 7
    z, w, s = _inputs(T, N, V, d, K, dtype, False, True, True, seed=4)
    p, head = vm.problem(T, N, d, 8, 1, 1, 1.0, dtype), vm.head_config(V, K, 2.0)
    least, most = vm.vmoe_head_min_workspace_size(p, head), vm.vmoe_head_workspace_size(p, head)
    assert 0 < least < most
    for nbytes in (least, (least + most) // 2, most):
        _check(_run(p, head, z, w, s, nbytes), z, w, s, 2.0, dtype)
    with pytest.raises(vm.VmoeError):
        _run(p, head, z, w, s, least - 1)


def test_gradients_one_at_a_time():
    T, N, V, d, K = 2, 130, 700, 128, 5
    z, w, s = _inputs(T, N, V, d, K, "bf16", True, True, True, seed=6)
    p, head = vm.problem(T, N, d, 8, 1, 1, 1.0, "bf16"), vm.head_config(V, K, 2.0, True)
    for only in ("dce", "dlse", "dkl"):
        one = dict(s, **{n: s[n] if n == only else None for n in ("dce", "dlse", "dkl")})
        _check(_run(p, head, z, w, one), z, w, one, 2.0, "bf16")
    both = _run(p, head, z, w, s)
    assert torch.equal(_run(p, head, z, w, s, train=False)["dz"], both["dz"])
    assert torch.equal(_run(p, head, z, w, s, dz=False)["dw"], both["dw"])


def test_nothing_to_learn_from():
    """No label and no teacher anywhere, in one task or in all: zeros, whatever lies in z and in the gradients."""
    T, N, V, d, K = 3, 70, 500, 64, 4
    z, w, s = _inputs(T, N, V, d, K, "bf16", False, True, False, seed=7)
    s["label"][1], s["tidx"][1] = -1, -1
    z[1] = float("nan")
    for n in ("dce", "dlse", "dkl"):
        s[n][1] = float("nan")
    p, head = vm.problem(T, N, d, 8, 1, 1, 1.0, "bf16"), vm.head_config(V, K, 2.0)
    o = _run(p, head, z, w, s)
    assert all(torch.all(o[n][1] == 0) for n in ("ce", "lse", "kl", "tlse", "logp", "dz", "dw"))
    s["label"][:], s["tidx"][:] = -1, -1
    o = _run(p, head, z, w, s)
    assert all(torch.all(o[n] == 0) for n in ("ce", "lse", "kl", "tlse", "logp", "dz", "dw"))


def test_wide_logits():
    """Logits of hundreds: losses of hundreds and of next to nothing."""
    T, N, V, d = 1, 200, 900, 64
    z, w, s = _inputs(T, N, V, d, 6, "bf16", False, True, False, seed=8)
    z = z * 40
    p, head = vm.problem(T, N, d, 8, 1, 1, 1.0, "bf16"), vm.head_config(V, 6, 2.0)
    r = _check(_run(p, head, z, w, s), z, w, s, 2.0, "bf16")
    assert r["ce"].max() > 100 and r["ce"].min() < 1e-3


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tau", [0.5, 1.0, 2.0])
@pytest.mark.parametrize("N", [40, 200])
def test_wide_logits_of_tokens_without_a_label_or_a_teacher(N, tau, dtype):
    """Logits of hundreds, a third of the tokens with a label alone, a third with a teacher alone, a third with both: all
    gradients together, each by itself, and each left out.  exp of a logit that nothing is taken from is infinite here.

    Of logits so wide many p lie at the end of fp32's range: an exponential below 2^-126 is 0 (ex2.approx.ftz), and its weight
    is below 1, so a dl of two of them is off by up to 2 * 2^-126; its parts and their products with z or w, where they are
    that small, by as much again: 2^-124 a dl, beside the relative bounds."""
    T, V, d, K = 2, 900, 64, 6
    z, w, s = _inputs(T, N, V, d, K, dtype, N == 200, True, False, seed=8)
    z = z * 40
    s["label"][:, 0::3], s["tidx"][:, 1::3] = -1, -1
    p, head = vm.problem(T, N, d, 8, 1, 1, 1.0, dtype), vm.head_config(V, K, tau, N == 200)
    r = ref.loss(z, w, s["label"], s["tidx"], s["tlogit"], tau)
    assert np.abs(r["logits"]).max(axis=(1, 2)).min() > 200 and (r["has"] != r["taught"]).mean() > 0.6
    for given in (("dce", "dlse", "dkl"), ("dce",), ("dlse",), ("dkl",), ("dce", "dkl"), ("dce", "dlse")):
        one = dict(s, **{n: s[n] if n in given else None for n in ("dce", "dlse", "dkl")})
        o = _run(p, head, z, w, one)
        assert torch.isfinite(o["dz"]).all() and torch.isfinite(o["dw"]).all(), given
        _check(o, z, w, one, tau, dtype, flushed=2.0 ** -124)


def test_stream_graph_and_two_at_once():
    T, N, V, d, K = 2, 150, 800, 128, 5
    cases = [_inputs(T, N, V, d, K, "bf16", False, True, True, seed=i) for i in (1, 2)]
    p, head = vm.problem(T, N, d, 8, 1, 1, 1.0, "bf16"), vm.head_config(V, K, 2.0)
    want = [_run(p, head, *c) for c in cases]
    names = ("ce", "lse", "kl", "tlse", "logp", "dz", "dw")
    z, w, s = cases[0]
    buf = [z.cuda(), w.cuda(), *(_dev(s[n]) for n in ("label", "tidx", "tlogit", "dce", "dlse", "dkl"))]
    ws = torch.empty(vm.vmoe_head_workspace_size(p, head), dtype=torch.uint8, device="cuda")
    o = {n: torch.full_like(want[0][n], float("nan")) for n in names}

    def step(stream=None):
        z, w, y, i, q, a, b, c = buf
        vm.vmoe_head_loss(p, head, z, w, y, i, q, o["ce"], o["lse"], o["kl"], o["tlse"], o["logp"], ws, stream=stream)
        vm.vmoe_head_loss_bwd(p, head, z, w, y, i, q, o["ce"], o["lse"], o["tlse"], o["logp"], a, b, c, o["dz"], o["dw"], ws,
                              stream=stream)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step()
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.synchronize()
    for k in (1, 0):
        z, w, s = cases[k]
        for b, v in zip(buf, [z, w, *(s[n] for n in ("label", "tidx", "tlogit", "dce", "dlse", "dkl"))]):
            b.copy_(v)
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):  # another call beside it
            other = _run(p, head, *cases[1 - k])
        torch.cuda.synchronize()
        for n in names:
            assert torch.equal(o[n], want[k][n]) and torch.equal(other[n], want[1 - k][n]), n


def _forward(p, head, z, w, s):
    T, N, K = p.T, p.N, head.teacher_k
    new = lambda *sh: torch.empty(sh, device="cuda")  # noqa: E731
    o = dict(ce=new(T, N), lse=new(T, N), kl=new(T, N) if K else None, tlse=new(T, N) if K else None,
             logp=new(T, N, K) if K else None)
    ws = torch.full((vm.vmoe_head_workspace_size(p, head),), 255, dtype=torch.uint8, device="cuda")
    vm.vmoe_head_loss(p, head, z.cuda(), w.cuda(), _dev(s["label"]), _dev(s["tidx"]), _dev(s["tlogit"]), o["ce"], o["lse"], o["kl"],
                      o["tlse"], o["logp"], ws)
    return o


@pytest.mark.parametrize("tau", (1.0, 2.0))
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("N", (5, 40))
def test_nan_token(N, dtype, tau):
    """A token of NaN that takes part: its losses are NaN, whichever kernel sums its logits; the others' stay."""
    p, head, T, V, d, K = vm.problem(2, N, 64, 8, 1, 1, 1.0, dtype), vm.head_config(300, 4, tau), 2, 300, 64, 4
    z, w, s = _inputs(T, N, V, d, K, dtype, False, True, False, seed=4)
    z[1, 3] = float("nan")
    o = _forward(p, head, z, w, s)
    bad = torch.zeros(T, N, dtype=torch.bool)
    bad[1, 3] = True
    for n in ("ce", "lse", "kl", "tlse"):
        assert torch.equal(torch.isnan(o[n]).cpu(), bad), n


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("size", [(1, 5, 90001, 40, 0, 1.0), (3, 16, 30010, 136, 9, 2.0), (1, 9, 700, 1032, 3, 0.5), (2, 2, 5000, 2048, 0, 1.0)],
                         ids=str)
def test_few_tokens(size, dtype):
    """At most 16 tokens: more entries than all warps take at a time, widths around what they are taken up to."""
    T, N, V, d, K, tau = size
    p, head = vm.problem(T, N, d, 8, 1, 1, 1.0, dtype), vm.head_config(V, K, tau)
    z, w, s = _inputs(T, N, V, d, K, dtype, False, True, True, seed=6)
    o = _forward(p, head, z, w, s)
    _check(o, z, w, dict(s, dce=None, dlse=None, dkl=None), tau, dtype)


@pytest.mark.parametrize("N", (5, 40))
def test_entries_out_of_reach(N):
    """Weights of -inf against tokens of positive values: logits of -inf, whole half tiles of them, add nothing."""
    T, V, d = 2, 600, 64
    p, head = vm.problem(T, N, d, 8, 1, 1, 1.0, "bf16"), vm.head_config(V)
    z, w, s = _inputs(T, N, V, d, 0, "bf16", False, True, False, seed=5)
    z = z.abs() + 1
    s["label"] = s["label"] % 100
    cut = torch.zeros(V, dtype=torch.bool)
    cut[128:256] = cut[500:] = True
    lost = w.clone()
    lost[:, cut] = float("-inf")
    o = _forward(p, head, z, lost, s)
    few = w[:, ~cut].contiguous()
    r = ref.loss(z, few, s["label"], None, None, 1.0)  # labels lie before what is cut out
    D = (d / 16 + 4) * 2.0 ** -23 * np.einsum("tnd,tvd->tnv", np64(z), np.abs(np64(few))).max(axis=2)
    assert np.all(np.abs(np64(o["lse"]) - r["lse"]) <= D + 1e-6 + 2.0 ** -23 * np.abs(r["lse"]))
    assert np.all(np.abs(np64(o["ce"]) - r["ce"]) <= 2 * D + 2e-6 + 2.0 ** -22 * np.abs(r["ce"]))


@pytest.mark.parametrize("size", [(1, 1, 700, 128, 0, 1.0), (2, 3, 5003, 72, 9, 2.0), (90, 16, 600, 264, 5, 1.0), (2, 17, 5003, 136, 9, 2.0),
                                  (1, 31, 700, 72, 0, 1.0), (3, 128, 2000, 64, 3, 1.0), (1, 97, 40000, 264, 4, 0.5)], ids=str)
def test_few_tokens_gradients(size):
    """At most 128 tokens a head: dl, of which few values make most of the gradient, is kept to 2^-16 in bf16 problems."""
    T, N, V, d, K, tau = size
    p, head = vm.problem(T, N, d, 8, 1, 1, 1.0, "bf16"), vm.head_config(V, K, tau)
    z, w, s = _inputs(T, N, V, d, K, "bf16", False, True, True, seed=7)
    _check(_run(p, head, z, w, s), z, w, s, tau, "bf16", few=True)
    _check(_run(p, head, z, w, s, vm.vmoe_head_min_workspace_size(p, head)), z, w, s, tau, "bf16", few=True)


@pytest.mark.parametrize("value", ["-inf", "lowest"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [5, 40, 150])
def test_entries_switched_off(N, dtype, value):
    """Weights of -inf, and of the type's lowest value, against tokens of positive values: losses and gradients are those of the
    other entries alone.  dz of bf16 weights of -inf is 0 times them, which the header leaves out."""
    T, V, d, K, tau = 2, 600, 64, 4, 2.0
    p, head = vm.problem(T, N, d, 8, 1, 1, 1.0, dtype), vm.head_config(V, K, tau)
    z, w, s = _inputs(T, N, V, d, K, dtype, False, True, False, seed=5)
    z = z.abs() + 1
    s["label"], s["tidx"] = s["label"] % 100, s["tidx"] % 100
    cut = torch.zeros(V, dtype=torch.bool)
    cut[128:256] = cut[500:] = True
    lost = w.clone()
    lost[:, cut] = float("-inf") if value == "-inf" else torch.finfo(w.dtype).min
    o = _run(p, head, z, lost, s, dz=dtype == "f32" or value == "lowest")
    assert torch.all(o["dw"][:, cut] == 0)
    _check(dict(o, dw=o["dw"][:, ~cut]), z, w[:, ~cut].contiguous(), s, tau, dtype, flushed=2.0 ** -124)


@pytest.mark.parametrize("tau", [30.0, 1e3, 1e6])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,K", [(40, 3), (150, 40)])
def test_high_temperatures(N, K, dtype, tau):
    """A model that is sure of an entry in the teacher's list that is not the label: its part of the gradient of ce does not pass
    through the logarithm at the temperature, whose roundings it would multiply."""
    T, V, d = 2, 700, 72
    z, w, s = _inputs(T, N, V, d, K, dtype, True, True, False, seed=9)
    s["tidx"][..., K - 1] = (s["label"] + 1) % V
    z = (z.double() + 6 * w.double()[s["tidx"][..., K - 1].long()]).to(w.dtype)
    p, head = vm.problem(T, N, d, 8, 1, 1, 1.0, dtype), vm.head_config(V, K, tau, True)
    for nbytes in (None, vm.vmoe_head_min_workspace_size(p, head)):
        r = _check(_run(p, head, z, w, s, nbytes), z, w, s, tau, dtype)
    at = np.take_along_axis(r["logits"], s["tidx"][..., K - 1:].numpy().astype(np.int64), 2)[..., 0]
    assert np.median(np.exp(at - r["lse"])) > 0.5


@pytest.mark.parametrize("size", [(1, 197, 1000, 384, 8, 2.0), (1, 129, 9001, 72, 0, 1.0), (1, 256, 5000, 264, 5, 0.5), (5, 193, 1500, 136, 0, 1.0)],
                         ids=str)
def test_gradients_of_an_image(size):
    """Up to 256 tokens a head against a small vocabulary, one image's as a rule: dl is kept to 2^-16 as well."""
    T, N, V, d, K, tau = size
    p, head = vm.problem(T, N, d, 8, 1, 1, 1.0, "bf16"), vm.head_config(V, K, tau)
    for ragged in (False, True):
        z, w, s = _inputs(T, N, V, d, K, "bf16", False, True, ragged, seed=7)
        _check(_run(p, head, z, w, s), z, w, s, tau, "bf16", few=True)
        _check(_run(p, head, z, w, s, vm.vmoe_head_min_workspace_size(p, head)), z, w, s, tau, "bf16", few=True)
