"""Transformer blocks around the expert layers: norms, gate, residual and the layer, several deep.

Plumbing only, like ``step.py``: torch allocates the buffers, the library's kernels compute.  A
block is z' = rho z + gate * norm(layer(norm(z))) (Section 2.1: the experts stand in the place of a
ViT block's MLP); the norm behind one layer, the residual and the norm ahead of the next one are one
call.
"""
from __future__ import annotations

import bisect

import torch

from . import (VMOE_NORM_POST, _stream, norm_config, vmoe_block_norm, vmoe_block_norm_bwd, vmoe_block_norm_bwd_workspace_size)
from .step import BalanceBuffers, Buffers, GateBuffers, StepRunner, _nothing_to_add_to

NORM_PARAMS = ("pre_w", "pre_b", "post_w", "post_b", "gate")


def _span(t):
    """The bytes of a contiguous tensor, from and to."""
    return t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()


class BlockStack:
    """L blocks of problem ``p``, forward and backward.

    ``layers``: for each block a dict of device tensors w_router, bias (or None), w1, w2 as for
    StepRunner, and of its norms' fp32 [T,d] parameters pre_w, pre_b, post_w, post_b, gate, each
    optional.  ``norm``: norm_config(...); post_* are used only if it has a norm on the branch.
    ``balance``: the balance losses' weights, see BalanceBuffers; each block computes its own.
    ``token_mask`` [T,N] uint8: 0 for padding that the losses leave out.  ``gating``: a VmoeGating
    (gating(...)) for experts that are chosen by vmoe_gate, each block with a bias of its own, in
    ``gates``, which ``update_gates(rate)`` moves; token_mask's padding then goes nowhere, but passes
    through the norms and has to be finite.

    ``forward(x)`` returns z [T,N,d]; ``backward(dz)`` returns dx and leaves every parameter's
    gradient in ``grads[l][name]``.  Both run on the current stream, or on ``stream``, and write the
    same buffers in every call: an ``x`` that lies in one of them (the z or dx of an earlier call, a
    layer's y) is refused, since the backward reads x again; give a copy.  So is a ``dz`` in the last
    layer's input gradient, which is written while dz is read; z and dx may be given.
    """

    def __init__(self, p, layers, norm=None, balance=None, token_mask=None, device="cuda", gating=None):
        if not layers:
            raise ValueError("a stack has at least one block")
        if _nothing_to_add_to(p, balance):
            raise ValueError("VMOE_DLOGITS_ADD without balance: no step writes the gradients that it adds to")
        self.p, self.layers = p, layers
        self.norm = norm if norm is not None else norm_config()
        self.post = bool(self.norm.flags & VMOE_NORM_POST)
        like = lambda t: None if t is None else torch.empty_like(t)  # noqa: E731
        stat = lambda: torch.empty((p.T, p.N, 2), dtype=torch.float32, device=device)  # noqa: E731
        self.runners, self.grads = [], []
        for w in layers:
            b = Buffers(p, device)
            inp = dict(x=torch.empty_like(b.y), dy=torch.empty_like(b.y), w_router=w["w_router"], bias=w.get("bias"),
                       w1=w["w1"], w2=w["w2"], token_mask=token_mask)
            r = StepRunner(p, inp, b, router_grad=True,
                           balance=None if balance is None else BalanceBuffers(p, balance, device),
                           gating=None if gating is None else GateBuffers(p, gating, device=device))
            self.runners.append(r)
            g = {n: like(self._par(w, n)) for n in NORM_PARAMS}
            g.update(w_router=b.dw_router, bias=None if w.get("bias") is None else b.dbias, w1=b.dw1, w2=b.dw2)
            self.grads.append(g)
        self.gates = [r.gating for r in self.runners]
        first = self.runners[0].b.y
        self.z = [torch.empty_like(first) for _ in layers]  # behind each block
        self.pre_stat = [stat() for _ in layers]
        self.post_stat = [stat() if self.post else None for _ in layers]
        self.dz = torch.empty_like(first)
        self.workspace = torch.empty(vmoe_block_norm_bwd_workspace_size(p), dtype=torch.uint8, device=device)
        self.x = None
        own = [*self.z, self.dz, self.workspace, *self.pre_stat, *self.post_stat]
        for r, g in zip(self.runners, self.grads):
            own += [*vars(r.b).values(), r.inp["x"], r.inp["dy"], *g.values()]
            own += [] if r.balance is None else [v for n, v in vars(r.balance).items() if n != "dloss"]
            own += [] if r.gating is None else [r.gating.select_bias, r.gating.demand, r.gating.workspace]
        self._own = sorted({_span(t) for t in own if isinstance(t, torch.Tensor)})

    def _par(self, layer, name):
        return layer.get(name) if self.post or not name.startswith("post") else None

    def _norm_args(self, block, after):
        """The parameters of the call between a block's layer and the next one's."""
        mine = [None] * 3 if block is None else [self._par(block, n) for n in ("post_w", "post_b", "gate")]
        return mine, [None] * 2 if after is None else [after.get("pre_w"), after.get("pre_b")]

    def forward(self, x, stream=None):
        beg, end = _span(x)
        last = bisect.bisect_left(self._own, (end, 0)) - 1  # the buffers do not overlap: the last that begins before x's end
        if last >= 0 and self._own[last][1] > beg:
            raise ValueError("x is a buffer of the stack, which its own calls overwrite: give a copy")
        p, stream = self.p, _stream(stream)
        self.x = x
        _, pre = self._norm_args(None, self.layers[0])
        vmoe_block_norm(p, self.norm, x, None, None, None, None, *pre, None, self.runners[0].inp["x"], None,
                        self.pre_stat[0], stream)
        z = x
        for i, r in enumerate(self.runners):
            r.forward(stream)
            last = i + 1 == len(self.runners)
            post, pre = self._norm_args(self.layers[i], None if last else self.layers[i + 1])
            vmoe_block_norm(p, self.norm, z, r.b.y, *post, *pre, self.z[i], None if last else self.runners[i + 1].inp["x"],
                            self.post_stat[i], None if last else self.pre_stat[i + 1], stream)
            z = self.z[i]
        return z

    def backward(self, dz, stream=None):
        if self.x is None:
            raise RuntimeError("backward before forward")
        beg, end = _span(dz)
        for t in (self.runners[-1].inp["dy"], self.dz):  # dx may be dz itself
            b, e = _span(t)
            if beg < e and b < end and not (t is self.dz and beg == b):
                raise ValueError("dz lies in a buffer that is written while it is read: give a copy")
        p, stream = self.p, _stream(stream)
        du = None
        for i in reversed(range(len(self.runners))):
            r, g = self.runners[i], self.grads[i]
            after = None if du is None else self.layers[i + 1]
            post, pre = self._norm_args(self.layers[i], after)
            ahead = {} if after is None else self.grads[i + 1]
            vmoe_block_norm_bwd(p, self.norm, r.b.y, None if du is None else self.z[i], self.post_stat[i],
                                None if du is None else self.pre_stat[i + 1], *post, pre[0], dz, du, self.dz, r.inp["dy"],
                                g["post_w"], g["post_b"], g["gate"], ahead.get("pre_w"), ahead.get("pre_b"),
                                self.workspace, stream=stream)
            r.backward(stream)
            dz, du = self.dz, r.b.dx
        g = self.grads[0]
        vmoe_block_norm_bwd(p, self.norm, None, self.x, None, self.pre_stat[0], None, None, None, self.layers[0].get("pre_w"),
                            dz, du, self.dz, None, None, None, None, g["pre_w"], g["pre_b"], self.workspace, stream=stream)
        return self.dz

    def balance_losses(self):
        """[T,3] losses of each block's last forward (see vmoe_balance), or None without them."""
        return [None if r.balance is None else r.balance.loss for r in self.runners]

    def update_gates(self, rate, stream=None):
        """Moves every block's selection bias towards an even demand, by ``rate`` (see vmoe_gate_bias)."""
        stream = _stream(stream)
        for gate in self.gates:
            if gate is not None:
                gate.update(rate, stream)

    def parameters(self):
        """A dict for each adapted tensor: name, param, grad, and decay: False for biases, norms and
        gates, which a weight decay leaves alone."""
        out = []
        for i, (w, g) in enumerate(zip(self.layers, self.grads)):
            for n in ("w1", "w2", "w_router", "bias") + NORM_PARAMS:
                if g.get(n) is not None:
                    out.append(dict(name="%d.%s" % (i, n), param=w[n], grad=g[n], decay=n in ("w1", "w2", "w_router")))
        return out
