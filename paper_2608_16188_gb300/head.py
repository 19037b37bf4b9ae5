"""What a stack of blocks is trained against: labels and a teacher's logits, through a head over a vocabulary.

Plumbing only, like ``step.py``: torch allocates the buffers, vmoe_head_loss and its backward compute.
"""
from __future__ import annotations

import torch

from . import (VMOE_HEAD_SHARED, _stream, head_config, vmoe_head_loss, vmoe_head_loss_bwd, vmoe_head_workspace_size)


class Head:
    """A head of problem ``p``'s tokens over the V entries of ``w`` [T,V,d], or [V,d] for one head for all
    tasks, in the problem's dtype.

    ``labels``: cross entropy against labels; ``teacher_k``, ``temperature``: distillation from a teacher's
    teacher_k logits a token.  ``train``: ``dw`` is the gradient of ``w``, which ``parameters()`` hands to an
    optimizer; without it the head is frozen.  ``workspace_bytes``: less than the recommended scratch, for less
    memory (see vmoe_head_min_workspace_size).

    ``forward`` leaves the losses [T,N] in ``ce`` and ``kl`` (and lse, tlse, logp as in vmoe_head_loss);
    ``backward`` returns dz [T,N,d].  Both write the same buffers in every call and run on the current stream, or on
    ``stream``; the tensors given to forward have to stay as they are until its backward has run."""

    def __init__(self, p, w, labels=True, teacher_k=0, temperature=1.0, train=True, workspace_bytes=None, device="cuda"):
        if w.dim() not in (2, 3):
            raise ValueError("a head's weights: [T, V, d], or [V, d] for one head for all tasks")
        if not labels and not teacher_k:
            raise ValueError("a head is trained against labels, a teacher, or both")
        self.p, self.w = p, w
        self.config = head_config(w.shape[-2], teacher_k, temperature, shared=w.dim() == 2)
        new = lambda have, *shape: torch.empty(shape, device=device) if have else None  # noqa: E731
        self.ce, self.lse = new(labels, p.T, p.N), new(labels, p.T, p.N)
        self.kl, self.tlse, self.logp = new(teacher_k, p.T, p.N), new(teacher_k, p.T, p.N), new(teacher_k, p.T, p.N, teacher_k)
        self.dz = torch.empty((p.T, p.N, p.d_model), dtype=w.dtype, device=device)
        self.dw = torch.empty_like(w) if train else None
        size = vmoe_head_workspace_size(p, self.config) if workspace_bytes is None else workspace_bytes
        self.workspace = torch.empty(size, dtype=torch.uint8, device=device)
        self.inputs = None

    @property
    def shared(self):
        return bool(self.config.flags & VMOE_HEAD_SHARED)

    def forward(self, z, label=None, teacher_idx=None, teacher_logit=None, stream=None):
        """Losses of tokens z [T,N,d]: label [T,N] int32 (outside [0, V): none), teacher_idx [T,N,K] int32
        (outside: left out) and teacher_logit [T,N,K] fp32.  Returns (ce, kl), None for what is not there."""
        self.inputs = None  # a call that is refused leaves nothing to go back through
        vmoe_head_loss(self.p, self.config, z, self.w, label, teacher_idx, teacher_logit, self.ce, self.lse, self.kl, self.tlse,
                       self.logp, self.workspace, stream=_stream(stream))
        self.inputs = (z, label, teacher_idx, teacher_logit)
        return self.ce, self.kl

    def backward(self, dce=None, dkl=None, dlse=None, stream=None):
        """dz for the gradients [T,N] fp32 of the losses (zero where None) of the last forward; dw with it."""
        if self.inputs is None:
            raise RuntimeError("backward before forward")
        z, label, teacher_idx, teacher_logit = self.inputs
        vmoe_head_loss_bwd(self.p, self.config, z, self.w, label, teacher_idx, teacher_logit, self.ce, self.lse, self.tlse,
                           self.logp, dce, dlse, dkl, self.dz, self.dw, self.workspace, stream=_stream(stream))
        return self.dz

    def parameters(self, name="head"):
        """The head's weights for an optimizer, as BlockStack.parameters(); empty for a frozen one."""
        return [] if self.dw is None else [dict(name=name, param=self.w, grad=self.dw, decay=True)]
