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
    below half a bf16 step are lost.
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

    def moments(self, i):
        """(m, v) of tensor i as fp32 values."""
        t = self.tensors[i]
        m, v = t["m"].float(), t["v"].float()
        if "m_scale" not in t:
            return m, v
        per = lambda s: s.repeat_interleave(256)[:m.numel()].view_as(m)  # noqa: E731
        return m * per(t["m_scale"]), (v * per(t["v_scale"])) ** 2
