"""What an adaptation step trains against and how its routers choose, as cases that can be timed and compared.

``head``     a head over a large vocabulary behind the blocks (vmoe_head_loss, vmoe_head_loss_bwd): softmax cross
             entropy against labels, without keeping the logits, as it evaluates ("fwd") or with its gradients
             into the tokens and, where the head is trained too, into its weights ("step").
``distill``  the same call against a teacher's largest logits at a temperature, with labels beside them or not.
``gate``     the choice of experts from router logits (vmoe_gate): softmax or sigmoid scores, a bias that balances
             the choice but not the gates, groups of experts, capacity slots; as it serves ("fwd") or with the
             gradient through the gates into the router (vmoe_gate_bwd, "step").

The sizes are those of ``workloads.py`` and of the tests, or generic: 197 tokens an image, vocabularies from a
thousand answers to the 128,000 entries of a large tokenizer.
"""
from __future__ import annotations

import math

import torch

own = False

DEFAULTS = dict(
    # T tasks of N tokens, width d
    T=1, N=197, d=384, dtype="bf16", mode="step",
    # head, distill: V entries, one head for all tasks (shared), its gradient (train), labels, K logits of the
    # teacher at temperature tau; "ragged": padded batches and tokens without a label or a teacher
    V=1000, shared=False, train=True, label=True, K=0, tau=1.0, mask="none",
    # gate: E experts a task, top-k, "sigmoid" | "softmax" scores, groups of which `kept` are open, each
    # scored by the sum of its `top` best; gates renormalised or not, times `scale`; capacity factor
    E=8, k=2, score="sigmoid", groups=1, kept=1, top=1, renorm=True, scale=1.0, cf=1.25)


def _case(op, **kw):
    return dict(DEFAULTS, op=op, **kw)


def listed():
    return [
        # one image's tokens against a thousand classes, evaluated: latency
        _case("head", name="head_1image_fwd", mode="fwd"),
        # a few tokens scored over a large tokenizer's vocabulary: the weights' bytes
        _case("head", name="head_4tokens_fwd", mode="fwd", N=4, d=1024, V=128000),
        # 17 tasks, a head each, trained with it: the ViT-B co-adaptation step
        _case("head", name="head_step_vitb_t17", T=17, N=8 * 197, d=768, V=32000),
        # one frozen head behind all tasks, half of whose tokens are padding or carry no label
        _case("head", name="head_step_frozen_padded", T=8, N=1024, d=1024, V=50304, shared=True, train=False,
              mask="ragged"),
        # an fp32 head of odd sizes
        _case("head", name="head_step_f32_odd", T=3, N=333, d=200, V=5003, dtype="f32"),
        # one image against a teacher's eight largest logits: latency
        _case("distill", name="distill_1image", K=8, label=False, tau=2.0),
        # labels and a teacher together, at another temperature, over the six-task step's tokens
        _case("distill", name="distill_labels_vitb_t6", T=6, N=16 * 197, d=768, V=16384, K=32, tau=2.0),
        # odd sizes, padding and short teacher lists
        _case("distill", name="distill_odd_padded", T=3, N=1001, d=384, V=10007, K=50, label=False, tau=4.0,
              mask="ragged"),
        # one image through one task's router, as it serves: latency
        _case("gate", name="gate_1image_fwd", mode="fwd"),
        # the 17-task step: sigmoid scores, four of eight groups open, with the router's gradient
        _case("gate", name="gate_step_vitb_t17", T=17, N=8 * 197, d=768, E=32, groups=8, kept=4, top=2, scale=2.5),
        # softmax scores without renormalisation, top-1 of 64, padded batches
        _case("gate", name="gate_step_softmax_padded", T=8, N=8 * 197, d=1024, E=64, k=1, score="softmax", renorm=False,
              cf=1.0, mask="ragged"),
        # long token streams over the most experts a task may have
        _case("gate", name="gate_long_fwd", mode="fwd", T=4, N=65536, E=256, k=8, groups=8, kept=4, top=2),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    op = rng.choice(["head", "distill", "gate"])
    most = 6.0 * 17 * 8 * 197 * 768 * 32000
    while True:
        mode, mask = rng.choice(["fwd", "step", "step"]), rng.choice(["none", "ragged"])
        if op != "gate":
            f32 = rng.random() < 0.25
            c = _case(op, mode=mode, mask=mask, T=_log(rng, 1, 17), N=_log(rng, 1, 4096), d=8 * _log(rng, 8, 128),
                      V=_log(rng, 500, 128000), shared=rng.random() < 0.4, train=rng.random() < 0.7,
                      dtype="f32" if f32 else "bf16")
            if op == "distill":
                c.update(K=_log(rng, 1, 100), label=rng.random() < 0.5, tau=rng.choice([1.0, 2.0, 2.0, 4.0, 0.5]))
            heads = 1 if c["shared"] else c["T"]
            if heads * c["V"] * c["d"] <= 17 * 32000 * 768 and work(c)["flops"] * (12 if f32 else 1) <= most:
                return c
        else:
            E = _log(rng, 1, 256)
            sizes = [g for g in (1, 1, 1, 2, 4, 8, 16) if E % g == 0]
            groups = rng.choice(sizes)
            kept = rng.randint(max(1, groups // 4), groups)
            c = _case(op, mode=mode, mask=mask, T=_log(rng, 1, 32), N=_log(rng, 1, 65536), d=8 * _log(rng, 8, 128), E=E,
                      k=min(8, kept * (E // groups), rng.choice([1, 2, 2, 4, 6, 8])), groups=groups, kept=kept,
                      top=min(rng.choice([1, 2]), E // groups), score=rng.choice(["sigmoid", "sigmoid", "softmax"]),
                      renorm=rng.random() < 0.7, scale=rng.choice([1.0, 1.0, 2.5]), cf=rng.choice([1.0, 1.25, 2.0]),
                      dtype=rng.choice(["bf16", "bf16", "f32"]))
            if c["T"] * E <= 1024 and work(c)["bytes"] <= 4.2 * 65536 * 256 * 4:
                return c


# ---------------------------------------------------------------------------------------------------
# What a pass cannot do without.


def _el(c):
    return 4 if c["dtype"] == "f32" else 2


def work(case):
    c = dict(DEFAULTS, **case)
    n = float(c["T"] * c["N"])
    if c["op"] == "gate":
        E, k, d = c["E"], c["k"], c["d"]
        nbytes = n * (4 * E + 12 * k + (c["mask"] != "none")) + 12.0 * c["T"] * E
        flops = 30.0 * n * E
        if c["mode"] == "step":  # x, dy, dx; the chosen rows of ye; dgate, dlogits; the router and its gradient
            rows = min(n * k, float(c["T"] * E * _capacity(c)))
            nbytes += n * d * _el(c) * 4 + rows * d * _el(c) + n * (4 * E + 4 * k) + 8.0 * c["T"] * E * (d + 1)
            flops += 2.0 * n * d * (k + 2 * E)
        return {"bytes": nbytes, "flops": flops}
    heads = 1 if c["shared"] else c["T"]
    rows = n * (0.5 if c["mask"] == "ragged" else 1.0)  # tokens that take part
    w = float(heads) * c["V"] * c["d"]
    products, nbytes = 1, rows * c["d"] * _el(c) + w * _el(c) + n * (12 + 12 * c["K"])
    if c["mode"] == "step":
        products += 1 + c["train"]
        nbytes += n * c["d"] * _el(c) + (w * _el(c) if c["train"] else 0) + n * 8
    return {"bytes": nbytes, "flops": 2.0 * products * rows * c["V"] * c["d"]}


# ---------------------------------------------------------------------------------------------------
# Inputs.


def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 6151 + 17)
    return g


def _capacity(c):
    return max(1, min(c["N"], math.ceil(c["cf"] * c["k"] * c["N"] / c["E"])))


def _takes_part(c, g):
    """[T,N]: the tokens in front of a task's length, half of the batch in the mean."""
    T, N = c["T"], c["N"]
    if c["mask"] == "none":
        return torch.ones((T, N), dtype=torch.bool, device="cuda")
    length = torch.randint(1, N + 1, (T, 1), generator=g, device="cuda")
    length[0] = N
    keep = torch.arange(N, device="cuda") < length
    return keep & (torch.rand((T, N), generator=g, device="cuda") < 0.9)  # a prompt's tokens carry no label


def _prepare_head(c, seed):
    g = _gen(seed)
    T, N, d, V, K, dt = c["T"], c["N"], c["d"], c["V"], c["K"], _dtype(c["dtype"])
    heads = 1 if c["shared"] else T
    rand = lambda *shape: torch.rand(shape, generator=g, device="cuda")  # noqa: E731
    w = torch.empty((heads, V, d), dtype=dt, device="cuda")
    for h in range(heads):  # logits of normalised tokens: a deviation of 1.5
        w[h] = 1.5 / math.sqrt(d) * torch.randn((V, d), generator=g, device="cuda")
    true = torch.randint(0, V, (T, N), generator=g, device="cuda")
    z = torch.randn((T, N, d), generator=g, device="cuda")
    for t in range(T):  # some tokens are sure of their answer, others are not
        z[t] += 5.0 * rand(N, 1) * w[0 if c["shared"] else t][true[t]].float()
    keep = _takes_part(c, g)
    z[~keep] = float("nan")  # padding holds anything
    s = dict(c=c, z=z.to(dt), w=w[0] if c["shared"] else w, label=None, tidx=None, tlogit=None)
    if c["label"]:
        label = torch.where(rand(T, N) < 0.8, true, torch.randint(0, V, (T, N), generator=g, device="cuda"))
        s["label"] = torch.where(keep, label, torch.full_like(label, -1)).to(torch.int32)
    if K:
        # the teacher's largest logits, in order, at K entries of which the first is the answer
        step = 1 + (rand(T, N, 1) * max(1, V // K - 1)).long().clamp(max=max(0, V // K - 1))
        tidx = (true[..., None] + step * torch.arange(K, device="cuda")) % V
        tlogit = 6.0 * rand(T, N, 1) - torch.cumsum(-torch.log(rand(T, N, K).clamp(min=1e-6)), 2)
        if c["mask"] == "ragged":  # a teacher that keeps what holds most of its mass
            short = torch.randint(1, K + 1, (T, N, 1), generator=g, device="cuda")
            tidx = torch.where(torch.arange(K, device="cuda") < short, tidx, torch.full_like(tidx, -1))
        s["tidx"] = torch.where(keep[..., None], tidx, torch.full_like(tidx, -1)).to(torch.int32)
        s["tlogit"] = tlogit
    s["dce"] = s["dkl"] = None
    if c["mode"] == "step":  # the mean over the tokens, some of them weighted
        each = (0.5 + rand(T, N)) / keep.sum()
        s["dce"] = each if c["label"] else None
        s["dkl"] = c["tau"] ** 2 * each if K else None  # the usual factor for a temperature
    if own:
        import paper_2608_16188_gb300 as vm
        s["p"] = vm.problem(T, N, d, 8, 1, 1, 1.0, c["dtype"])
        s["head"] = vm.head_config(V, teacher_k=K, temperature=c["tau"], shared=c["shared"])
        f32 = lambda *shape: torch.empty(shape, device="cuda")  # noqa: E731
        s["out"] = dict(ce=f32(T, N) if c["label"] else None, lse=f32(T, N) if c["label"] else None,
                        kl=f32(T, N) if K else None, tlse=f32(T, N) if K else None, logp=f32(T, N, K) if K else None)
        if c["mode"] == "step":
            s["grads"] = dict(dz=torch.empty_like(s["z"]), dw=torch.empty_like(s["w"]) if c["train"] else None)
        s["ws"] = torch.empty(vm.vmoe_head_workspace_size(s["p"], s["head"]), dtype=torch.uint8, device="cuda")
    return s


def _prepare_gate(c, seed):
    g = _gen(seed)
    T, N, E, d, k, dt = c["T"], c["N"], c["E"], c["d"], c["k"], _dtype(c["dtype"])
    randn = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    s = dict(c=c, mask=None)
    s["logits"] = randn(T, N, E) + 0.5 * randn(T, 1, E)  # drifted routers
    s["bias"] = (0.1 if c["score"] == "sigmoid" else 0.1 / E) * randn(T, E)
    if c["mask"] == "ragged":
        keep = _takes_part(c, g)
        s["mask"] = keep.to(torch.uint8)
        s["logits"][~keep] = float("nan")
        if E > 2 * k and c["groups"] == 1:  # an expert switched off
            s["logits"][:, :, E // 3] = float("-inf")
    C = _capacity(c)
    if c["mode"] == "step":
        s["x"] = randn(T, N, d).to(dt)
        s["w_router"] = randn(T, d, E) / math.sqrt(d)
        s["dy"] = randn(T, N, d).to(dt)
        s["ye"] = torch.empty((T, E, C, d), dtype=dt, device="cuda")
        for t in range(T):
            s["ye"][t] = randn(E, C, d)
        s["dx_in"] = randn(T, N, d).to(dt)  # the expert path's share
    if own:
        import paper_2608_16188_gb300 as vm
        s["p"] = vm.problem(T, N, d, 8, E, k, c["cf"], c["dtype"],
                            vm.VMOE_LOGITS_IN | (0 if c["renorm"] else vm.VMOE_NO_RENORM))
        s["gating"] = vm.gating(score=c["score"], groups=c["groups"], groups_kept=c["kept"], group_top=c["top"],
                                scale=c["scale"])
        i32, f32 = torch.int32, torch.float32
        new = lambda *shape, dtype=f32: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
        s["out"] = dict(idx=new(T, N, k, dtype=i32), gate=new(T, N, k), slot=new(T, N, k, dtype=i32),
                        load=new(T, E, dtype=i32), demand=new(T, E, dtype=i32))
        if c["mode"] == "step":
            s["grads"] = dict(dgate=new(T, N, k), dlogits=new(T, N, E), dw_router=new(T, d, E), dbias=new(T, E),
                              dx=torch.empty_like(s["x"]))
        s["ws"] = new(max(1, vm.vmoe_gate_workspace_size(s["p"])), dtype=torch.uint8)
    return s


def prepare(case, seed):
    c = dict(DEFAULTS, **case)
    return _prepare_gate(c, seed) if c["op"] == "gate" else _prepare_head(c, seed)


# ---------------------------------------------------------------------------------------------------
# The framework's calls.


def _own_head(s):
    import paper_2608_16188_gb300 as vm
    o = s["out"]
    vm.vmoe_head_loss(s["p"], s["head"], s["z"], s["w"], s["label"], s["tidx"], s["tlogit"], o["ce"], o["lse"], o["kl"],
                      o["tlse"], o["logp"], s["ws"])
    if s["c"]["mode"] == "fwd":
        return o
    d = s["grads"]
    vm.vmoe_head_loss_bwd(s["p"], s["head"], s["z"], s["w"], s["label"], s["tidx"], s["tlogit"], o["ce"], o["lse"],
                          o["tlse"], o["logp"], s["dce"], None, s["dkl"], d["dz"], d["dw"], s["ws"])
    return dict(o, **d)


def _own_gate(s):
    import paper_2608_16188_gb300 as vm
    o = s["out"]
    vm.vmoe_gate(s["p"], s["gating"], None, None, None, s["bias"], s["mask"], s["logits"], o["idx"], o["gate"], o["slot"],
                 o["load"], o["demand"], s["ws"])
    if s["c"]["mode"] == "fwd":
        return o
    d = s["grads"]
    vm.vmoe_gate_bwd(s["p"], s["gating"], s["x"], s["w_router"], s["logits"], o["idx"], o["gate"], o["slot"], s["dy"],
                     s["ye"], d["dgate"], d["dlogits"], d["dw_router"], d["dbias"], s["dx_in"], d["dx"])
    return dict(o, **d)


# ---------------------------------------------------------------------------------------------------
# The plain forms.


def _plain_teacher(tidx, tlogit, V, tau):
    """The teacher's distribution over the entries that count, which those are, and its logarithm."""
    on = (tidx >= 0) & (tidx < V) & (tlogit != float("-inf"))
    some = on.any(1, keepdim=True)
    t = torch.where(on, tlogit / tau, torch.full_like(tlogit, float("-inf")))
    top = torch.where(some, t.amax(1, keepdim=True), torch.zeros_like(t[:, :1]))
    e = torch.exp(t - top)
    total = torch.where(some, e.sum(1, keepdim=True), torch.ones_like(top))
    logq = torch.where(on, t - top - torch.log(total), torch.zeros_like(t))
    return e / total, logq, on, some[:, 0]


def _plain_lse(logits):
    top = logits.amax(1, keepdim=True)
    return (top + torch.log(torch.exp(logits - top).sum(1, keepdim=True)))[:, 0]


def _plain_head(s):
    c = s["c"]
    T, N, d, V, K, tau = c["T"], c["N"], c["d"], c["V"], c["K"], c["tau"]
    step = c["mode"] == "step"
    flat = (1, T * N) if c["shared"] else (T, N)  # heads, tokens of a head
    w_all = s["w"].reshape(flat[0], V, d)
    outs = {n: [] for n in ("ce", "lse", "kl", "tlse", "logp", "dz", "dw")}
    for h in range(flat[0]):
        at = lambda t, *tail: None if t is None else t.reshape(*flat, *tail)[h]  # noqa: E731
        label, tidx, tlogit = at(s["label"]), at(s["tidx"], K), at(s["tlogit"], K)
        has = torch.zeros(flat[1], dtype=torch.bool, device="cuda")
        taught = has
        if label is not None:
            has = (label >= 0) & (label < V)
        if K:
            q, logq, on, taught = _plain_teacher(tidx, tlogit, V, tau)
        part = has | taught
        zero = torch.zeros(flat[1], device="cuda")
        z = torch.where(part[:, None], at(s["z"], d).float(), torch.zeros((), device="cuda"))
        w = w_all[h].float()
        logits = z @ w.t()
        dl = None
        if label is not None:
            lse = _plain_lse(logits)
            pick = torch.where(has, label, torch.zeros_like(label)).long()[:, None]
            outs["lse"].append(torch.where(has, lse, zero))
            outs["ce"].append(torch.where(has, lse - logits.gather(1, pick)[:, 0], zero))
            if step:
                each = torch.where(has, at(s["dce"]), zero)[:, None]
                dl = torch.exp(logits - lse[:, None]) * each
                dl.scatter_add_(1, pick, -each)
        if K:
            soft = logits / tau
            tlse = _plain_lse(soft)
            entry = torch.where(on, tidx, torch.zeros_like(tidx)).long()
            logp = torch.where(on, soft.gather(1, entry) - tlse[:, None], torch.zeros_like(tlogit))
            outs["tlse"].append(torch.where(taught, tlse, zero))
            outs["logp"].append(logp)
            outs["kl"].append(torch.where(taught, (q * (logq - logp)).sum(1), zero))
            if step:
                each = torch.where(taught, at(s["dkl"]) / tau, zero)[:, None]
                more = torch.exp(soft - tlse[:, None]) * each
                more.scatter_add_(1, entry, -each * q * on)
                dl = more if dl is None else dl + more
        if step:
            outs["dz"].append((dl @ w).to(s["z"].dtype))
            if c["train"]:
                outs["dw"].append((dl.t() @ z).to(s["w"].dtype))
    shape = dict(ce=(T, N), lse=(T, N), kl=(T, N), tlse=(T, N), logp=(T, N, K), dz=(T, N, d), dw=tuple(s["w"].shape))
    out = {n: torch.stack(v).reshape(shape[n]) if v else None for n, v in outs.items()}
    return out if step else {n: out[n] for n in ("ce", "lse", "kl", "tlse", "logp")}


def _plain_choice(s):
    """Scores and choice in 64 bits, for one choice next to another's score decides whole numbers; [T,N,E]."""
    c = s["c"]
    T, N, E = c["T"], c["N"], c["E"]
    x = s["logits"].double()
    off = torch.isnan(x) | (x == float("-inf"))
    if s["mask"] is not None:
        off = off | (s["mask"] == 0)[..., None]
    low = torch.full_like(x, float("-inf"))
    x = torch.where(off, low, x)
    if c["score"] == "sigmoid":
        score = 1.0 / (1.0 + torch.exp(-x))
    else:
        top = x.amax(2, keepdim=True)
        e = torch.exp(x - torch.where(top == float("-inf"), torch.zeros_like(top), top))
        score = e / e.sum(2, keepdim=True).clamp(min=1e-300)
    value = torch.where(off, low, score + s["bias"].double()[:, None, :])
    if c["groups"] > 1:
        g = value.view(T, N, c["groups"], E // c["groups"])
        best = g.sort(dim=3, descending=True).values[..., :c["top"]].sum(3)
        order = best.sort(dim=2, descending=True, stable=True).indices[..., :c["kept"]]
        shut = torch.ones_like(best, dtype=torch.bool).scatter_(2, order, False)
        value = torch.where(shut[..., None], low.view_as(g), g).view(T, N, E)
    return score, value


def _plain_slots(idx, E, C):
    """Choice by choice, in token order: the place of each assignment among its expert's; load; demand."""
    T, N, k = idx.shape
    seq = idx.transpose(1, 2).reshape(T, k * N).long()
    seq = torch.where(seq < 0, torch.full_like(seq, E), seq)
    order = seq.sort(dim=1, stable=True)
    count = torch.zeros((T, E + 1), dtype=torch.long, device="cuda").scatter_add_(1, seq, torch.ones_like(seq))
    start = torch.cumsum(count, 1) - count
    place = torch.arange(k * N, device="cuda")[None, :] - start.gather(1, order.values)
    rank = torch.empty_like(place).scatter_(1, order.indices, place)
    slot = torch.where((rank < C) & (seq < E), rank, torch.full_like(rank, -1))
    demand = count[:, :E].to(torch.int32)
    return slot.view(T, k, N).transpose(1, 2).to(torch.int32).contiguous(), demand.clamp(max=C), demand


def _plain_gate(s):
    c = s["c"]
    T, N, E, k, d = c["T"], c["N"], c["E"], c["k"], c["d"]
    score, value = _plain_choice(s)
    order = value.sort(dim=2, descending=True, stable=True)
    idx = order.indices[..., :k]
    there = order.values[..., :k] != float("-inf")
    chosen = torch.where(there, score.gather(2, idx), torch.zeros((), dtype=torch.float64, device="cuda"))
    mass = chosen.sum(2, keepdim=True)
    share = chosen / torch.where(mass > 0, mass, torch.ones_like(mass)) if c["renorm"] else chosen
    gate = (c["scale"] * share).float()
    idx = torch.where(there, idx, torch.full_like(idx, -1)).to(torch.int32)
    slot, load, demand = _plain_slots(idx, E, _capacity(c))
    o = dict(idx=idx, gate=gate, slot=slot, load=load, demand=demand)
    if c["mode"] == "fwd":
        return o
    dt = s["x"].dtype
    kept = slot >= 0
    e, at = idx.clamp(min=0).long(), slot.clamp(min=0).long()
    dy = s["dy"].float()
    dgate = torch.empty((T, N, k), device="cuda")
    for t in range(T):
        for j in range(k):
            dgate[t, :, j] = (dy[t] * s["ye"][t, e[t, :, j], at[t, :, j]].float()).sum(1)
    dgate = torch.where(kept, dgate, torch.zeros_like(dgate))
    p, sh = chosen.float(), share.float()
    mean = (sh * dgate).sum(2, keepdim=True)
    if c["score"] == "sigmoid":
        dsel = c["scale"] * sh * (1.0 - p) * (dgate - mean if c["renorm"] else dgate)
        dense = torch.zeros((T, N, E), device="cuda")
    elif c["renorm"]:
        dsel = c["scale"] * sh * (dgate - mean)
        dense = torch.zeros((T, N, E), device="cuda")
    else:
        dsel = c["scale"] * p * dgate
        dense = -c["scale"] * mean * score.float()
    dlogits = dense.scatter_add(2, e, torch.where(there, dsel, torch.zeros_like(dsel)))
    x, w = s["x"].float(), s["w_router"]
    dx = (s["dx_in"].float() + dlogits @ w.transpose(1, 2)).to(dt)
    return dict(o, dgate=dgate, dlogits=dlogits, dw_router=x.transpose(1, 2) @ dlogits, dbias=dlogits.sum(1), dx=dx)


def run(state):
    gate = state["c"]["op"] == "gate"
    if own:
        return _own_gate(state) if gate else _own_head(state)
    return _plain_gate(state) if gate else _plain_head(state)


# ---------------------------------------------------------------------------------------------------
# The definitions in 64 bits.


def _exact_head(s):
    c = s["c"]
    T, N, d, V, K, tau = c["T"], c["N"], c["d"], c["V"], c["K"], c["tau"]
    names = ("ce", "lse", "kl", "tlse", "logp") + (("dz", "dw") if c["mode"] == "step" else ())
    f64 = dict(dtype=torch.float64, device="cuda")
    o = dict.fromkeys(names)
    if c["label"]:
        o["ce"], o["lse"] = torch.zeros((T, N), **f64), torch.zeros((T, N), **f64)
    if K:
        o["kl"], o["tlse"], o["logp"] = torch.zeros((T, N), **f64), torch.zeros((T, N), **f64), torch.zeros((T, N, K), **f64)
    if c["mode"] == "step":
        o["dz"] = torch.zeros((T, N, d), **f64)
        if c["train"]:
            o["dw"] = torch.zeros(tuple(s["w"].shape), **f64)
    for t in range(T):
        w = (s["w"] if c["shared"] else s["w"][t]).double()
        for lo in range(0, N, 1024):
            n = torch.arange(lo, min(N, lo + 1024), device="cuda")
            used = torch.zeros(len(n), dtype=torch.bool, device="cuda")
            if c["label"]:
                used |= (s["label"][t, n] >= 0) & (s["label"][t, n] < V)
            if K:
                used |= ((s["tidx"][t, n] >= 0) & (s["tidx"][t, n] < V) & ~torch.isneginf(s["tlogit"][t, n])).any(1)
            n = n[used]
            if len(n) == 0:
                continue
            z = s["z"][t, n].double()
            logit = torch.einsum("nd,vd->nv", z, w)
            grad = torch.zeros_like(logit) if c["mode"] == "step" else None
            if c["label"]:
                y = s["label"][t, n].long()
                r = torch.arange(len(n), device="cuda")[(y >= 0) & (y < V)]
                logp = torch.log_softmax(logit[r], 1)
                o["lse"][t, n[r]] = torch.logsumexp(logit[r], 1)
                o["ce"][t, n[r]] = -logp[torch.arange(len(r)), y[r]]
                if grad is not None:
                    g = torch.exp(logp)
                    g[torch.arange(len(r)), y[r]] -= 1.0
                    grad[r] += s["dce"][t, n[r]].double()[:, None] * g
            if K:
                i = s["tidx"][t, n].long()
                ok = (i >= 0) & (i < V) & ~torch.isneginf(s["tlogit"][t, n])
                r = torch.arange(len(n), device="cuda")[ok.any(1)]
                i, ok = i[r].clamp(0, V - 1), ok[r]
                logq = torch.log_softmax((s["tlogit"][t, n[r]].double() / tau).masked_fill(~ok, float("-inf")), 1)
                q = torch.exp(logq)
                full = torch.log_softmax(logit[r] / tau, 1)
                mine = torch.take_along_dim(full, i, 1).masked_fill(~ok, 0.0)
                o["logp"][t, n[r]] = mine
                o["tlse"][t, n[r]] = torch.logsumexp(logit[r] / tau, 1)
                o["kl"][t, n[r]] = (q * (logq.masked_fill(~ok, 0.0) - mine)).sum(1)
                if grad is not None:
                    g = torch.exp(full)
                    g.scatter_add_(1, i, -q)
                    grad[r] += s["dkl"][t, n[r]].double()[:, None] / tau * g
            if grad is not None:
                o["dz"][t, n] = torch.einsum("nv,vd->nd", grad, w)
                if c["train"]:
                    dw = torch.einsum("nv,nd->vd", grad, z)
                    if c["shared"]:
                        o["dw"] += dw
                    else:
                        o["dw"][t] += dw
    return o


def _exact_gate(s):
    c = s["c"]
    T, N, E, k = c["T"], c["N"], c["E"], c["k"]
    first = _plain_gate(dict(s, c=dict(c, mode="fwd")))  # the whole numbers, which everything else follows
    out = dict.fromkeys(("idx", "slot", "load", "demand"))
    gates, more = [], {n: [] for n in ("dgate", "dlogits", "dw_router", "dbias", "dx")}
    for t in range(T):
        x = torch.nan_to_num(s["logits"][t].double(), nan=float("-inf"), posinf=float("inf"), neginf=float("-inf"))
        idx, slot = first["idx"][t].long(), first["slot"][t].long()
        on = idx >= 0
        prob = torch.sigmoid(x) if c["score"] == "sigmoid" else torch.nan_to_num(torch.softmax(x, 1))
        mine = torch.take_along_dim(prob, idx.clamp(min=0), 1) * on
        total = mine.sum(1, keepdim=True) if c["renorm"] else torch.ones((N, 1), dtype=torch.float64, device="cuda")
        part = torch.where(total > 0, mine / total, torch.zeros_like(mine))
        gates.append(c["scale"] * part)
        if c["mode"] == "fwd":
            continue
        ye, dy = s["ye"][t], s["dy"][t].double()
        dg = torch.zeros((N, k), dtype=torch.float64, device="cuda")
        for j in range(k):
            r = torch.nonzero(slot[:, j] >= 0)[:, 0]
            dg[r, j] = torch.einsum("nd,nd->n", dy[r], ye[idx[r, j], slot[r, j]].double())
        # by the scores, then by the logits
        dscore = torch.zeros((N, E), dtype=torch.float64, device="cuda")
        by = dg - (part * dg).sum(1, keepdim=True) if c["renorm"] else dg
        by = torch.where(total > 0, c["scale"] * by / total, torch.zeros_like(by)) * on
        dscore.scatter_add_(1, idx.clamp(min=0), by)
        if c["score"] == "sigmoid":
            dl = dscore * prob * (1.0 - prob)
        else:
            dl = prob * (dscore - (prob * dscore).sum(1, keepdim=True))
        more["dgate"].append(dg)
        more["dlogits"].append(dl)
        more["dw_router"].append(torch.einsum("nd,ne->de", s["x"][t].double(), dl))
        more["dbias"].append(dl.sum(0))
        more["dx"].append(s["dx_in"][t].double() + torch.einsum("ne,de->nd", dl, s["w_router"][t].double()))
    out["gate"] = torch.stack(gates)
    out = {n: out[n] for n in ("idx", "gate", "slot", "load", "demand")}
    return dict(out, **{n: torch.stack(v) for n, v in more.items()}) if c["mode"] == "step" else out


def exact(case, seed):
    c = dict(DEFAULTS, **case)
    s = prepare(case, seed)
    return _exact_gate(s) if c["op"] == "gate" else _exact_head(s)
