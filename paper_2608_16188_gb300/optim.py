"""AdamW over the tensors of an adaptation step: the states and the call (vmoe_adamw)."""
from __future__ import annotations

import torch

from . import _stream, adamw_tensors, vmoe_adamw


class AdamW:
    """AdamW with decoupled weight decay, one launch for all tensors (up to 380).

    ``params``: dicts with param and grad (contiguous device tensors that stay where they are, such
    as BlockStack.parameters() or a Buffers' gradients), and optionally lr_scale (1), decay (True)
    or weight_decay (this one instead of the common one).
    ``eight_bit``: moments of tensors of at least ``eight_bit_from`` elements in 8 bits.
    ``master``: an fp32 copy of bf16 parameters, which the updates work on; without it updates
    below half a bf16 step are lost.  The parameters are written from it: call
    ``refresh_master`` after loading others into them.
    ``capturable``: the step number is counted on the device, so that ``step`` may be captured
    into a CUDA graph and replayed; ``lr_factor`` [1], a device tensor that the learning rate is
    taken times, is then the way to change it.
    """

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, eight_bit=False,
                 eight_bit_from=4096, master=True, seed=0, capturable=False):
        self.lr, self.betas, self.eps, self.seed = lr, betas, eps, seed
        self.steps = 0
        self.tensors = []
        for d in params:
            p = d["param"]
            n, dev = p.numel(), p.device
            t = dict(param=p, grad=d["grad"], lr_scale=d.get("lr_scale", 1.0),
                     weight_decay=d.get("weight_decay", weight_decay if d.get("decay", True) else 0.0))
            eight = eight_bit and n >= eight_bit_from
            kind = torch.float8_e4m3fn if eight else torch.float32
            t["m"], t["v"] = (torch.zeros(p.shape, dtype=kind, device=dev) for _ in range(2))
            if eight:
                t["m_scale"], t["v_scale"] = (torch.zeros((n + 255) // 256, device=dev) for _ in range(2))
            if master and p.dtype == torch.bfloat16:
                t["master"] = p.detach().float()
            self.tensors.append(t)
        self.table = adamw_tensors(self.tensors)
        self.step_dev = self.lr_factor = None
        if capturable:
            device = self.tensors[0]["param"].device if self.tensors else "cuda"
            self.step_dev = torch.zeros(1, dtype=torch.int32, device=device)
            self.lr_factor = torch.ones(1, device=device)

    def step(self, grad_scale=None, stream=None):
        """One update from the gradients.  ``grad_scale``: a [1] fp32 device tensor that they are
        taken times; one that is infinite or NaN leaves everything as it was but for the step's
        number.  ``stream``: a torch.cuda.Stream, or None for the current one."""
        if self.step_dev is None:
            vmoe_adamw(self.table, self.steps + 1, self.lr, *self.betas, self.eps, self.seed, grad_scale=grad_scale,
                       stream=_stream(stream))
        else:  # counted behind the call: one that is refused leaves the number as it was
            vmoe_adamw(self.table, 1, self.lr, *self.betas, self.eps, self.seed, self.step_dev, self.lr_factor, grad_scale,
                       stream=_stream(stream))
            with torch.cuda.stream(stream):
                self.step_dev.add_(1)
        self.steps += 1

    def refresh_master(self, stream=None):
        """Takes the master copies from the parameters again, after something else than ``step`` wrote them."""
        with torch.cuda.stream(stream):
            for t in self.tensors:
                if t.get("master") is not None:
                    t["master"].copy_(t["param"].detach())

    STATE = ("m", "v", "m_scale", "v_scale", "master")

    def state_dict(self):
        """What a later run needs to go on, beside the parameters: the step's number, the seed of the 8-bit moments'
        rounding, and each tensor's moments, scales and master copy (the arrays themselves, not copies)."""
        out = dict(step=self.steps if self.step_dev is None else int(self.step_dev), seed=self.seed,
                   tensors=[{k: t[k] for k in self.STATE if t.get(k) is not None} for t in self.tensors])
        if self.lr_factor is not None:
            out["lr_factor"] = float(self.lr_factor)
        return out

    def load_state_dict(self, state):
        """Goes on from ``state``, of an AdamW over tensors of the same sizes in the same order, with the same kinds of
        moments.  Written in place, so that captured graphs see it (their seed stays theirs)."""
        theirs = state["tensors"]
        if len(theirs) != len(self.tensors):
            raise ValueError("a state of %d tensors for %d" % (len(theirs), len(self.tensors)))
        for i, (t, s) in enumerate(zip(self.tensors, theirs)):
            mine = {k: (tuple(t[k].shape), t[k].dtype) for k in self.STATE if t.get(k) is not None}
            if mine != {k: (tuple(v.shape), v.dtype) for k, v in s.items()}:
                raise ValueError("tensor %d: a state of other sizes, moments or master copies" % i)
        for t, s in zip(self.tensors, theirs):
            for k, v in s.items():
                t[k].copy_(v)
        self.steps, self.seed = int(state["step"]), state["seed"]
        if self.step_dev is not None:
            self.step_dev.fill_(self.steps)
            self.lr_factor.fill_(state.get("lr_factor", 1.0))

    def moments(self, i):
        """(m, v) of tensor i as fp32 values."""
        t = self.tensors[i]
        m, v = t["m"].float(), t["v"].float()
        if "m_scale" not in t:
            return m, v
        per = lambda s: s.repeat_interleave(256)[:m.numel()].view_as(m)  # noqa: E731
        return m * per(t["m_scale"]), (v * per(t["v_scale"])) ** 2
