"""The operators around the expert layer of an adaptation step, as cases that can be timed and compared.

``balance``  the routers' balance losses with per-expert counts (vmoe_balance) and their gradient into
             the logits (vmoe_balance_bwd): one call of each is one pass.
``norm``     the block around the layer, z = rho x + gate * norm(y), u = norm(z) (vmoe_block_norm), as
             it serves images ("fwd") or with its gradients (vmoe_block_norm_bwd, "step").
``adamw``    the update of many tensors at once (vmoe_adamw), its moments in fp32 or in 8 bits.

The sizes are those of ``workloads.py`` and of the tests, or generic ViT shapes (197 tokens an image).
"""
from __future__ import annotations

import math

import torch

own = False

DEFAULTS = dict(
    # balance, norm: T tasks of N tokens, width d, E experts a task, top-k
    T=1, N=197, d=384, E=8, k=2, dtype="bf16",
    # balance: "none", or "ragged": padded batches, with experts switched off by a logit of -inf
    mask="none", bias="none",
    # norm: "fwd" | "step"; part "pre" (u = norm(x)), "post" (z only) or "both"; post: a norm on y
    mode="step", part="both", rms=False, post=True, rho=1.0,
    # adamw: `tensors` of about `numel` elements each (odd: not a multiple of anything), `state`
    # "f32" | "8bit", gradients in `grad`, an fp32 master copy of bf16 parameters
    tensors=1, numel=1 << 20, odd=False, state="f32", grad="bf16", master=False)


def _case(op, **kw):
    return dict(DEFAULTS, op=op, **kw)


def listed():
    return [
        # one image through one task's layer: latency
        _case("balance", name="balance_1image"),
        # the 17-task ViT-B co-adaptation step
        _case("balance", name="balance_vitb_t17", T=17, N=8 * 197, E=32, bias="drift"),
        # skewed routers on padded batches, a few experts switched off
        _case("balance", name="balance_skew_padded", T=8, N=8 * 197, E=64, k=1, bias="zipf", mask="ragged"),
        # long token streams over the most experts a task may have
        _case("balance", name="balance_long", T=4, N=65536, E=256, k=8, bias="drift"),
        # one image through one block, as it serves: the norm ahead of the layer alone
        _case("norm", name="norm_1image_pre", mode="fwd", part="pre"),
        # the 17-task step: the norm behind one layer, its gate and residual, and the next layer's norm
        _case("norm", name="norm_step_vitb_t17", T=17, N=8 * 197, d=768),
        # large batches as they are served
        _case("norm", name="norm_fwd_vitl", mode="fwd", T=8, N=32 * 197, d=1024, post=False),
        # an fp32 block of an odd width, root-mean-square norms and a scaled residual
        _case("norm", name="norm_step_f32_odd", T=3, N=1001, d=1000, dtype="f32", rms=True, rho=1.4142),
        # routers, their biases, gates and norms of a small model: many small fp32 tensors, latency
        _case("adamw", name="adamw_small", tensors=40, numel=6000, odd=True, dtype="f32", grad="f32"),
        # the ViT-S experts of four tasks with fp32 moments and master weights
        _case("adamw", name="adamw_vits_t4", tensors=2, numel=4 * 8 * 384 * 1536, master=True),
        # many experts' weights as tensors of their own, of odd sizes, moments in 8 bits
        _case("adamw", name="adamw_8bit_many", tensors=192, numel=147000, odd=True, state="8bit"),
        # ViT-B experts of two tasks, moments in 8 bits: memory for more tasks on a card
        _case("adamw", name="adamw_8bit_vitb_t2", tensors=2, numel=2 * 32 * 768 * 3072, state="8bit"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    op = rng.choice(["balance", "norm", "adamw", "adamw"])
    while True:
        if op == "balance":
            E = _log(rng, 1, 256)
            c = _case(op, T=_log(rng, 1, 32), N=_log(rng, 1, 65536), E=E, k=min(E, rng.choice([1, 2, 2, 3, 4, 8])),
                      bias=rng.choice(["none", "drift", "zipf"]), mask=rng.choice(["none", "ragged"]))
            if c["T"] * E <= 1024 and c["T"] * c["N"] * E <= 4 * 65536 * 256:
                return c
        elif op == "norm":
            c = _case(op, T=_log(rng, 1, 32), N=_log(rng, 1, 8192), d=8 * _log(rng, 4, 256),
                      dtype=rng.choice(["bf16", "bf16", "f32"]), mode=rng.choice(["fwd", "step"]),
                      part=rng.choice(["pre", "post", "both", "both"]), rms=rng.random() < 0.4,
                      post=rng.random() < 0.6, rho=rng.choice([1.0, 1.0, 1.4142, 0.5]))
            if c["T"] * c["N"] * c["d"] <= 8 * 32 * 197 * 1024:
                return c
        else:
            bf16 = rng.random() < 0.75
            c = _case(op, tensors=_log(rng, 1, 300), numel=_log(rng, 1000, 1 << 27), odd=rng.random() < 0.6,
                      dtype="bf16" if bf16 else "f32", grad="f32" if not bf16 or rng.random() < 0.2 else "bf16",
                      state=rng.choice(["f32", "8bit"]), master=bf16 and rng.random() < 0.4)
            if c["tensors"] * c["numel"] <= 1 << 28:
                return c


# ---------------------------------------------------------------------------------------------------
# What a pass cannot do without.


def _el(c):
    return 4 if c["dtype"] == "f32" else 2


def work(case):
    c = dict(DEFAULTS, **case)
    if c["op"] == "balance":  # the logits in, their gradient out; the choices; the mask
        n = c["T"] * c["N"]
        return {"bytes": n * (8 * c["E"] + 4 * c["k"] + (c["mask"] != "none")) + 20.0 * c["T"] * c["E"],
                "flops": 14.0 * n * c["E"]}
    if c["op"] == "norm":
        n = float(c["T"] * c["N"] * c["d"])
        tensors = {"pre": 2, "post": 3, "both": 4}[c["part"]]  # x, y in; z, u out
        flops = 16.0
        if c["mode"] == "step":  # what came out again, its gradients in; the gradients of x, y out
            tensors += {"pre": 2, "post": 3, "both": 4}[c["part"]]
            flops = 48.0
        return {"bytes": n * _el(c) * tensors + 4.0 * 12 * c["T"] * c["d"], "flops": n * flops}
    n = float(sum(_sizes(c)))
    state = 16 if c["state"] == "f32" else 4 + 16 / 256
    return {"bytes": n * (2 * _el(c) + (4 if c["grad"] == "f32" else 2) + state + 8 * c["master"]), "flops": 20.0 * n}


# ---------------------------------------------------------------------------------------------------
# Inputs.


def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 11)
    return g


def _prepare_balance(c, seed):
    g = _gen(seed)
    T, N, E, k = c["T"], c["N"], c["E"], c["k"]
    logits = torch.randn((T, N, E), generator=g, device="cuda")
    if c["bias"] == "drift":
        logits += 0.5 * torch.randn((T, 1, E), generator=g, device="cuda")
    elif c["bias"] == "zipf":
        rank = torch.rand((T, 1, E), generator=g, device="cuda").argsort(dim=2)
        logits -= 1.2 * torch.log(rank + 1.0)
    mask = None
    if c["mask"] == "ragged":
        if E > k:  # one expert a task switched off
            off = torch.randint(0, E, (T, 1, 1), generator=g, device="cuda")
            logits.masked_fill_(torch.arange(E, device="cuda") == off, float("-inf"))
        idx = logits.topk(k, dim=2).indices.to(torch.int32).contiguous()
        length = torch.randint(0, N + 1, (T, 1), generator=g, device="cuda")
        length[0] = N
        keep = torch.arange(N, device="cuda") < length
        logits[~keep] = float("nan")  # padding holds anything
        idx[~keep] = -1
        mask = keep.to(torch.uint8)
        if N > 1:
            logits[0, N // 2] = float("-inf")  # a token that may go nowhere
    else:
        idx = logits.topk(k, dim=2).indices.to(torch.int32).contiguous()
    s = dict(c=c, logits=logits, idx=idx, mask=mask)
    s["dloss"] = torch.rand((T, 3), generator=g, device="cuda") * torch.tensor([0.02, 0.02, 0.002], device="cuda")
    if own:
        import paper_2608_16188_gb300 as vm
        s["p"] = vm.problem(T, N, 8, 8, E, k, 1.0, "f32")
        i32, f32 = torch.int32, torch.float32
        new = lambda *shape, dtype=f32: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
        s["out"] = dict(count=new(T, E, dtype=i32), tokens=new(T, dtype=i32), excess=new(T, E), loss=new(T, 3),
                        dlogits=new(T, N, E))
        s["ws"] = new(max(1, vm.vmoe_balance_workspace_size(s["p"])), dtype=torch.uint8)
    return s


def _prepare_norm(c, seed):
    g = _gen(seed)
    T, N, d, dt = c["T"], c["N"], c["d"], _dtype(c["dtype"])
    randn = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    s = dict(c=c, y=None, post_w=None, post_b=None, gate=None, pre_w=None, pre_b=None, dz=None, du=None)
    # a residual stream: channels with means of their own, some of them large
    s["x"] = (randn(T, N, d) + randn(T, 1, d).square()).to(dt)
    if c["part"] != "pre":
        s["y"] = (2.0 * randn(T, N, d) + 0.3).to(dt)
        s["gate"] = 0.5 + 0.2 * randn(T, d)
        if c["post"]:
            s["post_w"] = 1.0 + 0.1 * randn(T, d)
            s["post_b"] = None if c["rms"] else 0.1 * randn(T, d)
    if c["part"] != "post":
        s["pre_w"] = 1.0 + 0.1 * randn(T, d)
        s["pre_b"] = None if c["rms"] else 0.1 * randn(T, d)
    if c["mode"] == "step":
        s["dz"] = randn(T, N, d).to(dt)
        if c["part"] != "post":
            s["du"] = randn(T, N, d).to(dt)
    if own:
        import paper_2608_16188_gb300 as vm
        s["p"] = vm.problem(T, N, d, 8, 1, 1, 1.0, c["dtype"])
        s["cfg"] = vm.norm_config(rms=c["rms"], post=c["post"], eps=1e-6, residual_scale=c["rho"])
        like = lambda have, ref: torch.empty_like(ref) if have else None  # noqa: E731
        stat = lambda have: torch.empty((T, N, 2), device="cuda") if have else None  # noqa: E731
        step = c["mode"] == "step"
        s["out"] = dict(z=like(c["part"] != "pre", s["x"]), u=like(c["part"] != "post", s["x"]))
        s["post_stat"] = stat(step and c["part"] != "pre" and c["post"])
        s["pre_stat"] = stat(step and c["part"] != "post")
        if step:
            s["grads"] = dict(dx=torch.empty_like(s["x"]), dy=like(s["y"] is not None, s["x"]))
            for n in ("post_w", "post_b", "gate", "pre_w", "pre_b"):
                s["grads"]["d" + n] = like(s[n] is not None, s[n])
            s["ws"] = torch.empty(max(1, vm.vmoe_block_norm_bwd_workspace_size(s["p"])), dtype=torch.uint8,
                                  device="cuda")
    return s


LR, BETA1, BETA2, EPS, DECAY, SEED = 2e-4, 0.9, 0.999, 1e-8, 0.05, 1234


def _sizes(c):
    """Elements of each tensor: `numel`, or odd numbers around it."""
    n = c["numel"]
    if not c["odd"]:
        return [n] * c["tensors"]
    return [max(1, (n * (1 + (7 * i) % 13) // 7) | 1) for i in range(c["tensors"])]


def _prepare_adamw(c, seed):
    """Tensors in one flat buffer, each from a multiple of 256 elements on: the blocks of the 8-bit moments."""
    g = _gen(seed)
    sizes = _sizes(c)
    blocks = [-(-n // 256) for n in sizes]
    nb = sum(blocks)
    first = [sum(blocks[:i]) for i in range(len(blocks))] if len(blocks) < 400 else None
    tensor = torch.repeat_interleave(torch.arange(len(sizes), device="cuda"), torch.tensor(blocks, device="cuda"))
    begin = torch.tensor(first, device="cuda")[tensor]
    within = (torch.arange(nb, device="cuda") - begin).to(torch.int32)  # block number within its tensor
    size = torch.tensor(sizes, device="cuda")[tensor]
    keep = (within.long() * 256)[:, None] + torch.arange(256, device="cuda") < size[:, None]
    randn = lambda: torch.randn((nb, 256), generator=g, device="cuda")  # noqa: E731
    each = lambda lo, hi: torch.exp(torch.empty(len(sizes), device="cuda").uniform_(math.log(lo), math.log(hi), generator=g))[tensor][:, None]  # noqa: E731
    scale = each(1e-4, 1e-2)  # gradients differ between layers
    s = dict(c=c, sizes=sizes, blocks=blocks, first=first, tensor=tensor, within=within, step=10)
    param = 0.03 * randn() * keep
    s["param"] = param.to(_dtype(c["dtype"]))
    s["master"] = param if c["master"] else None
    quiet = torch.rand((nb, 1), generator=g, device="cuda") < 0.05  # experts that got no token
    s["grad"] = (scale * randn() * keep * ~quiet).to(_dtype(c["grad"]))
    m, root = 0.3 * scale * randn() * keep, scale * (0.2 + torch.rand((nb, 256), generator=g, device="cuda")) * keep
    if c["state"] == "f32":
        s["m"], s["v"], s["m_scale"], s["v_scale"] = m, root * root, None, None
    else:  # m and sqrt(v) as e4m3 values of a scale for each block
        s["m_scale"], s["v_scale"] = m.abs().amax(1) / 448, root.amax(1) / 448
        s["m"] = (m / s["m_scale"].clamp(min=1e-30)[:, None]).to(torch.float8_e4m3fn)
        s["v"] = (root / s["v_scale"].clamp(min=1e-30)[:, None]).to(torch.float8_e4m3fn)
    # no decay on every third tensor, half the rate on every fourth
    s["decay"] = [0.0 if i % 3 == 2 else DECAY for i in range(len(sizes))]
    s["rate"] = [0.5 if i % 4 == 3 else 1.0 for i in range(len(sizes))]
    s["grad_scale"] = torch.full((1,), 0.75, device="cuda")
    s["decay_of"] = torch.tensor(s["decay"], device="cuda")
    s["rate_of"] = torch.tensor(s["rate"], device="cuda")
    if own:
        import paper_2608_16188_gb300 as vm
        at = lambda t, i, n: None if t is None else t.view(-1)[256 * first[i]:256 * first[i] + n]  # noqa: E731
        sc = lambda t, i: None if t is None else t[first[i]:first[i] + blocks[i]]  # noqa: E731
        s["table"] = vm.adamw_tensors([
            dict(param=at(s["param"], i, n), grad=at(s["grad"], i, n), m=at(s["m"], i, n), v=at(s["v"], i, n),
                 m_scale=sc(s["m_scale"], i), v_scale=sc(s["v_scale"], i), master=at(s["master"], i, n),
                 lr_scale=s["rate"][i], weight_decay=s["decay"][i]) for i, n in enumerate(sizes)])
    return s


def prepare(case, seed):
    c = dict(DEFAULTS, **case)
    return {"balance": _prepare_balance, "norm": _prepare_norm, "adamw": _prepare_adamw}[c["op"]](c, seed)


# ---------------------------------------------------------------------------------------------------
# The framework's calls.


def _own_balance(s):
    import paper_2608_16188_gb300 as vm
    o = s["out"]
    vm.vmoe_balance(s["p"], s["logits"], s["idx"], s["mask"], o["count"], o["tokens"], o["excess"], o["loss"], s["ws"])
    vm.vmoe_balance_bwd(s["p"], s["logits"], s["mask"], o["count"], o["tokens"], o["excess"], s["dloss"], o["dlogits"])
    return o


def _own_norm(s):
    import paper_2608_16188_gb300 as vm
    o = s["out"]
    vm.vmoe_block_norm(s["p"], s["cfg"], s["x"], s["y"], s["post_w"], s["post_b"], s["gate"], s["pre_w"], s["pre_b"],
                       o["z"], o["u"], s["post_stat"], s["pre_stat"])
    if s["c"]["mode"] == "fwd":
        return o
    d = s["grads"]
    z = s["x"] if s["y"] is None else o["z"]
    vm.vmoe_block_norm_bwd(s["p"], s["cfg"], s["y"], z, s["post_stat"], s["pre_stat"], s["post_w"], s["post_b"],
                           s["gate"], s["pre_w"], s["dz"], s["du"], d["dx"], d["dy"], d["dpost_w"], d["dpost_b"],
                           d["dgate"], d["dpre_w"], d["dpre_b"], s["ws"])
    return dict(o, **d)


def _own_adamw(s):
    import paper_2608_16188_gb300 as vm
    s["step"] += 1
    vm.vmoe_adamw(s["table"], s["step"], LR, BETA1, BETA2, EPS, seed=SEED, grad_scale=s["grad_scale"])
    return _adamw_outputs(s)


def _adamw_outputs(s):
    # 8-bit moments: the e4m3 values, and the scale of each block of 256 that they are to be taken times
    return {n: s[n] for n in ("param", "master", "m", "v", "m_scale", "v_scale")}


# ---------------------------------------------------------------------------------------------------
# The plain forms.


def _plain_balance(s):
    c, logits, idx = s["c"], s["logits"], s["idx"]
    T, N, E, k = c["T"], c["N"], c["E"], c["k"]
    keep = torch.ones((T, N), dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"] != 0
    x = torch.where(keep[..., None], logits, torch.zeros_like(logits))
    top = x.amax(2, keepdim=True)
    keep = keep & (top[..., 0] != float("-inf"))  # nowhere to go: as padding
    top = torch.where(keep[..., None], top, torch.zeros_like(top))
    e = torch.exp(x - top)
    total = e.sum(2, keepdim=True)
    live = keep[..., None].to(torch.float32)
    prob = torch.where(keep[..., None], e / total, torch.zeros_like(e))
    lse = torch.where(keep, (top + torch.log(total))[..., 0], torch.zeros_like(live[..., 0]))
    tokens = keep.sum(1, dtype=torch.int32)
    into = torch.where(keep[..., None], idx, torch.full_like(idx, E)).reshape(T, -1).long()
    count = torch.zeros((T, E + 1), dtype=torch.int32, device="cuda")
    count = count.scatter_add_(1, into, torch.ones_like(into, dtype=torch.int32))[:, :E].contiguous()
    excess = (prob - live / E).sum(1, dtype=torch.float64)
    m = tokens.double().clamp(min=1)[:, None]
    some = (tokens > 0).double()[:, None]
    cf = count.double()
    all_choices = cf.sum(1, keepdim=True)
    loss = torch.cat([all_choices / (k * m) + E / (k * m * m) * (cf * excess).sum(1, keepdim=True),
                      E / (m * m) * (excess * excess).sum(1, keepdim=True),
                      lse.double().square().sum(1, keepdim=True) / m], dim=1) * some
    dl = s["dloss"].double()
    coef = (dl[:, 0:1] * E / (k * m * m) * (cf - all_choices / E) + dl[:, 1:2] * 2 * E / (m * m) * excess).float()[:, None, :]
    zc = (dl[:, 2:3] * 2 / m).float()[:, None, :]
    mean = (prob * coef).sum(2, keepdim=True)
    dlogits = prob * (coef - mean + zc * lse[..., None])
    return dict(count=count, tokens=tokens, excess=excess.float(), loss=loss.float(), dlogits=dlogits)


def _plain_norm_of(v, w, b, rms):
    """norm(v), (v - mean) * rstd, rstd."""
    if not rms:
        v = v - v.mean(2, keepdim=True)
    rstd = 1.0 / torch.sqrt(v.square().mean(2, keepdim=True) + 1e-6)
    hat = v * rstd
    out = hat * w[:, None, :]
    return out if b is None else out + b[:, None, :], hat, rstd


def _plain_norm_bwd(dout, w, hat, rstd, rms):
    dh = dout * w[:, None, :]
    r = dh - hat * (dh * hat).mean(2, keepdim=True)
    if not rms:
        r = r - dh.mean(2, keepdim=True)
    return r * rstd


def _plain_norm(s):
    c = s["c"]
    dt, rms, step = _dtype(c["dtype"]), c["rms"], c["mode"] == "step"
    o = dict(z=None, u=None)
    z = s["x"]
    if s["y"] is not None:
        w = hat = s["y"].float()
        if c["post"]:
            w, hat, rstd = _plain_norm_of(hat, s["post_w"], s["post_b"], rms)
        z = o["z"] = (c["rho"] * s["x"].float() + s["gate"][:, None, :] * w).to(dt)
    if c["part"] != "post":
        u, zhat, zrstd = _plain_norm_of(z.float(), s["pre_w"], s["pre_b"], rms)  # of z as it is stored
        o["u"] = u.to(dt)
    if not step:
        return o
    d = dict(dx=None, dy=None, dpost_w=None, dpost_b=None, dgate=None, dpre_w=None, dpre_b=None)
    dz = s["dz"].float()
    if s["du"] is not None:
        du = s["du"].float()
        dz = dz + _plain_norm_bwd(du, s["pre_w"], zhat, zrstd, rms)
        d["dpre_w"] = (du * zhat).sum(1)
        d["dpre_b"] = None if s["pre_b"] is None else du.sum(1)
    if s["y"] is None:
        d["dx"] = dz.to(dt)
        return dict(o, **d)
    d["dx"] = (c["rho"] * dz).to(dt)
    d["dgate"] = (dz * w).sum(1)
    dw = dz * s["gate"][:, None, :]
    if c["post"]:
        d["dpost_w"] = (dw * hat).sum(1)
        d["dpost_b"] = None if s["post_b"] is None else dw.sum(1)
        dw = _plain_norm_bwd(dw, s["post_w"], hat, rstd, rms)
    d["dy"] = dw.to(dt)
    return dict(o, **d)


def _signed(v):
    v &= 0xffffffff
    return v - (1 << 32) if v >> 31 else v


def _plain_dither(s):
    """Two 16-bit numbers an element: a hash of the seed, the step, the tensor's place and the element's."""
    lane = torch.arange(256, dtype=torch.int32, device="cuda")
    h = (s["within"][:, None] * 256 + lane) * _signed(0x51f6db5b)
    h = h + (s["tensor"] * 0x5e4087b3 & 0xffffffff).to(torch.int32)[:, None]
    h = h + _signed(SEED * 0xe32a5e87 + s["step"] * 0x339cd49b)
    h = (h ^ ((h >> 16) & 0xffff)) * _signed(0x9e4a8af7)
    h = (h ^ ((h >> 15) & 0x1ffff)) * _signed(0xa6bd2c99)
    h = h ^ ((h >> 16) & 0xffff)
    return h & 0xffff, (h >> 16) & 0xffff


def _plain_e4m3(v, bits, least):
    """(e4m3 values, scale of each block): v / scale rounded up or down to a neighbour, by `bits`."""
    top = v.abs().amax(1, keepdim=True)
    top = torch.where(top >= least, top, torch.zeros_like(top))
    inv = torch.where(top > 0, 448.0 / top, torch.zeros_like(top))
    a = v.abs() * inv
    low = torch.where(a < 2.0 ** -6, torch.full_like(a, 2.0 ** -6), torch.zeros_like(a))  # subnormals: one grid
    cut = ((a + low).view(torch.int32) + (bits * 16 + 8)) & -(1 << 20)  # three bits of the mantissa stay
    a = (cut.view(torch.float32) - low).clamp(max=448.0)
    return torch.where(v < 0, -a, a).to(torch.float8_e4m3fn), top[:, 0] / 448.0


def _plain_adamw(s):
    c = s["c"]
    s["step"] += 1
    g = s["grad"].float() * s["grad_scale"]
    p = (s["param"] if s["master"] is None else s["master"]).float()
    eight = c["state"] == "8bit"
    if eight:
        m = s["m"].float() * s["m_scale"][:, None]
        v = (s["v"].float() * s["v_scale"][:, None]).square()
    else:
        m, v = s["m"], s["v"]
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * (g * g)
    root = torch.sqrt(v)
    rate = (LR * s["rate_of"])[s["tensor"]][:, None]
    decay = s["decay_of"][s["tensor"]][:, None]
    c1, c2 = 1 - BETA1 ** s["step"], 1 - BETA2 ** s["step"]
    p = p * (1 - rate * decay) - rate * (m / c1) / (root / math.sqrt(c2) + EPS)
    s["param"].copy_(p)
    if s["master"] is not None:
        s["master"].copy_(p)
    if eight:
        lo, hi = _plain_dither(s)
        m, m_scale = _plain_e4m3(m, lo, 2.0 ** -100)
        v, v_scale = _plain_e4m3(root, hi, 2.0 ** -100)
        s["m_scale"].copy_(m_scale)
        s["v_scale"].copy_(v_scale)
    s["m"].copy_(m)
    s["v"].copy_(v)
    return _adamw_outputs(s)


def run(state):
    op = state["c"]["op"]
    if own:
        return {"balance": _own_balance, "norm": _own_norm, "adamw": _own_adamw}[op](state)
    return {"balance": _plain_balance, "norm": _plain_norm, "adamw": _plain_adamw}[op](state)


# ---------------------------------------------------------------------------------------------------
# The definitions in 64 bits.


def _exact_balance(s):
    c = s["c"]
    T, N, E, k = c["T"], c["N"], c["E"], c["k"]
    out = {n: [] for n in ("excess", "loss", "dlogits")}
    for t in range(T):
        x = s["logits"][t].double()
        on = torch.ones(N, dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"][t].bool()
        on = on & ~torch.isneginf(x).all(1)
        x = x[on]
        m = x.shape[0]
        d = torch.zeros((N, E), dtype=torch.float64, device="cuda")
        if m == 0:
            out["excess"].append(d.new_zeros(E))
            out["loss"].append(d.new_zeros(3))
            out["dlogits"].append(d)
            continue
        lse = torch.logsumexp(x, 1)
        prob = torch.exp(x - lse[:, None])
        count = torch.bincount(s["idx"][t][on].reshape(-1).long(), minlength=E).double()
        importance = prob.sum(0)
        out["excess"].append(importance - m / E)
        out["loss"].append(torch.stack([E / (k * m * m) * (count * importance).sum(),
                                        E / (m * m) * (importance - m / E).square().sum(), lse.square().mean()]))
        d0, d1, d2 = s["dloss"][t].double()
        dprob = d0 * E / (k * m * m) * count + d1 * 2 * E / (m * m) * importance
        d[on] = prob * (dprob - (prob * dprob).sum(1, keepdim=True)) + d2 * 2 / m * lse[:, None] * prob
        out["dlogits"].append(d)
    return dict({n: torch.stack(v) for n, v in out.items()}, count=None, tokens=None)


def _exact_norm(s):
    c = s["c"]
    n = lambda t: None if t is None else t.double()  # noqa: E731
    row = lambda t: 1.0 if t is None else t.double()[:, None, :]  # noqa: E731

    def stats(v):
        mu = 0.0 if c["rms"] else v.mean(2, keepdim=True)
        return mu, ((v - mu).square().mean(2, keepdim=True) + 1e-6).rsqrt()

    def back(v, mu, r, g):  # the derivative of sum(g * (v - mu) * r) by v
        h = (v - mu) * r
        t = g - h * (g * h).mean(2, keepdim=True)
        return r * (t if c["rms"] else t - g.mean(2, keepdim=True))

    x, y = n(s["x"]), n(s["y"])
    o = dict(z=None, u=None)
    z = x
    if y is not None:
        mu, r = stats(y) if c["post"] else (0.0, 1.0)
        h = (y - mu) * r
        w = h * row(s["post_w"]) + (0.0 if s["post_b"] is None else row(s["post_b"]))
        o["z"] = c["rho"] * x + row(s["gate"]) * w
        z = o["z"].to(s["x"].dtype).double()  # what follows sees the stored value
    if c["part"] != "post":
        zmu, zr = stats(z)
        zh = (z - zmu) * zr
        o["u"] = zh * row(s["pre_w"]) + (0.0 if s["pre_b"] is None else row(s["pre_b"]))
    if c["mode"] == "fwd":
        return o
    d = dict.fromkeys(("dx", "dy", "dpost_w", "dpost_b", "dgate", "dpre_w", "dpre_b"))
    dz, du = n(s["dz"]), n(s["du"])
    if du is not None:
        dz = dz + back(z, zmu, zr, du * row(s["pre_w"]))
        d["dpre_w"] = (du * zh).sum(1)
        d["dpre_b"] = None if s["pre_b"] is None else du.sum(1)
    if y is None:
        d["dx"] = dz
        return dict(o, **d)
    d["dx"] = c["rho"] * dz
    d["dgate"] = (dz * w).sum(1)
    dw = dz * row(s["gate"])
    if c["post"]:
        d["dpost_w"] = (dw * h).sum(1)
        d["dpost_b"] = None if s["post_b"] is None else dw.sum(1)
        dw = back(y, mu, r, dw * row(s["post_w"]))
    d["dy"] = dw
    return dict(o, **d)


def _exact_adamw(s):
    c, t = s["c"], s["step"] + 1
    outs = {n: [] for n in ("param", "m", "v", "m_scale", "v_scale")}
    nb = s["param"].shape[0]
    for lo in range(0, nb, 1 << 18):  # 64 M elements at a time
        at = slice(lo, min(nb, lo + (1 << 18)))
        g = s["grad"][at].double() * 0.75
        p = (s["param"] if s["master"] is None else s["master"])[at].double()
        m, v = s["m"][at].double(), s["v"][at].double()
        if c["state"] == "8bit":
            m, v = m * s["m_scale"][at].double()[:, None], (v * s["v_scale"][at].double()[:, None]) ** 2
        m, v = m + (1 - BETA1) * (g - m), v + (1 - BETA2) * (g * g - v)
        lr = LR * s["rate_of"].double()[s["tensor"][at]][:, None]
        wd = s["decay_of"].double()[s["tensor"][at]][:, None]
        adam = (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)).sqrt() + EPS)
        outs["param"].append(p - lr * (wd * p + adam))
        if c["state"] == "f32":
            outs["m"].append(m)
            outs["v"].append(v)
            continue
        # the hash in 64-bit integers
        e = s["within"][at].long()[:, None] * 256 + torch.arange(256, device="cuda")
        cut = lambda a: a & 0xffffffff  # noqa: E731
        h = cut(e * 0x51f6db5b + s["tensor"][at][:, None] * 0x5e4087b3 + (SEED * 0xe32a5e87 + t * 0x339cd49b) % (1 << 32))
        mul = lambda a, b: cut(a * (b & 0xffff) + (cut(a * (b >> 16)) << 16))  # noqa: E731
        h = mul(h ^ (h >> 16), 0x9e4a8af7)
        h = mul(h ^ (h >> 15), 0xa6bd2c99)
        h = h ^ (h >> 16)
        for name, value, r in (("m", m, h & 0xffff), ("v", v.sqrt(), h >> 16)):
            scale = value.abs().amax(1, keepdim=True) / 448
            a = (value / scale.clamp(min=1e-300)).abs()
            grid = torch.exp2(torch.frexp(a)[1].double().sub(1).clamp(min=-6) - 3)
            q = (grid * torch.floor(a / grid + (r.double() * 16 + 8) / (1 << 20))).clamp(max=448)
            outs[name].append(torch.copysign(q, value).float())
            outs[name + "_scale"].append(scale[:, 0])
    out = {n: torch.cat(v) if v else None for n, v in outs.items()}
    return dict(out, master=out["param"] if c["master"] else None)


def exact(case, seed):
    c = dict(DEFAULTS, **case)
    s = prepare(case, seed)
    return {"balance": _exact_balance, "norm": _exact_norm, "adamw": _exact_adamw}[c["op"]](s)
