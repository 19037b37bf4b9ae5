"""fp64 oracle of the losses behind the blocks (vmoe_head_loss, vmoe_head_loss_bwd), in numpy.

The formulas are those of include/vmoe.h; the paper (Section 3.1, Section 5.1) adapts the visual module to answers and
to a teacher's outputs and prints none.  Shares no code with the CUDA path.
"""
from __future__ import annotations

import numpy as np


def _np(a):
    return np.asarray(a.detach().cpu().double().numpy() if hasattr(a, "detach") else a, np.float64)


def _int(a):
    return np.asarray(a.cpu().numpy() if hasattr(a, "cpu") else a, np.int64)


def _lse(x):
    top = x.max(axis=-1)
    return top + np.log(np.exp(x - top[..., None]).sum(axis=-1))


def loss(z, w, label=None, tidx=None, tlogit=None, tau=1.0):
    """Outputs of vmoe_head_loss, and what the gradient needs: logits, q, which tokens have a label or a teacher.

    w [T,V,d], or [V,d] for one head for all tasks.  Rows of z without a part may hold anything."""
    z, w = _np(z), _np(w)
    T, N, d = z.shape
    w = np.broadcast_to(w, (T,) + w.shape) if w.ndim == 2 else w
    V = w.shape[1]
    r = dict(has=np.zeros((T, N), bool), taught=np.zeros((T, N), bool))
    if label is not None:
        y = _int(label)
        r["has"] = (y >= 0) & (y < V)
    if tidx is not None:
        i, t = _int(tidx), _np(tlogit)
        on = (i >= 0) & (i < V) & ~np.isneginf(t)
        r["taught"] = on.any(axis=2)
    part = r["has"] | r["taught"]
    l = np.einsum("tnd,tvd->tnv", np.where(part[..., None], z, 0.0), w)
    r["logits"] = l
    if label is not None:
        lse = _lse(l)
        r["lse"] = np.where(r["has"], lse, 0.0)
        r["ce"] = np.where(r["has"], lse - np.take_along_axis(l, np.where(r["has"], y, 0)[..., None], 2)[..., 0], 0.0)
    if tidx is not None:
        tl = np.where(on, t / tau, -np.inf)
        top = np.where(r["taught"], tl.max(axis=2), 0.0)[..., None]
        e = np.exp(tl - top)
        total = np.where(r["taught"], e.sum(axis=2), 1.0)[..., None]
        r["q"] = e / total
        logq = np.where(on, tl - top - np.log(total), 0.0)
        tlse = _lse(l / tau)
        r["logp"] = np.where(on, np.take_along_axis(l, np.where(on, i, 0), 2) / tau - tlse[..., None], 0.0)
        r["tlse"] = np.where(r["taught"], tlse, 0.0)
        r["kl"] = (r["q"] * (logq - r["logp"])).sum(axis=2)
    return r


def dlogits(r, label=None, tidx=None, tau=1.0, dce=None, dlse=None, dkl=None):
    """(dl, the sum of the magnitudes of its terms): the gradient by the logits."""
    l = r["logits"]
    T, N, V = l.shape
    dl, size = np.zeros_like(l), np.zeros_like(l)
    at = np.arange(T)[:, None, None], np.arange(N)[None, :, None]
    if label is not None:
        a = np.zeros((T, N)) if dce is None else np.where(r["has"], _np(dce), 0.0)
        b = np.zeros((T, N)) if dlse is None else np.where(r["has"], _np(dlse), 0.0)
        p = np.exp(l - np.where(r["has"], r["lse"], _lse(l))[..., None])
        dl += (a + b)[..., None] * p
        size += np.abs(a + b)[..., None] * p
        y = np.where(r["has"], _int(label), 0)[..., None]
        np.subtract.at(dl, at + (y,), a[..., None])
        np.add.at(size, at + (y,), np.abs(a)[..., None])
    if tidx is not None and dkl is not None:
        c = np.where(r["taught"], _np(dkl) / tau, 0.0)[..., None]
        p = np.exp(l / tau - _lse(l / tau)[..., None])
        dl += c * p
        size += np.abs(c) * p
        i = np.where(r["q"] > 0, _int(tidx), 0)
        np.subtract.at(dl, at + (i,), c * r["q"])
        np.add.at(size, at + (i,), np.abs(c) * r["q"])
    return dl, size


def back(dl, z, w, part):
    """dz and dw (summed over the tasks for one head)."""
    z, w = np.where(part[..., None], _np(z), 0.0), _np(w)
    wt = np.broadcast_to(w, (z.shape[0],) + w.shape) if w.ndim == 2 else w
    dw = np.einsum("tnv,tnd->tvd", dl, z)
    return np.einsum("tnv,tvd->tnd", dl, wt), dw.sum(axis=0) if w.ndim == 2 else dw
