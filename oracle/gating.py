"""fp64 oracle of the choice of experts by scores, bias and groups (vmoe_gate, vmoe_gate_bwd), in numpy.

Section 2.1 of the paper routes tokens to their most relevant experts under capacity limits (Challenge #1 in Section 1)
and assigns them one after another (Section 3.3.1); it gives no formula.  The reading is that of include/vmoe.h.
Shares no code with the CUDA path.
"""
from __future__ import annotations

import numpy as np


def _np(a):
    return None if a is None else np.asarray(a.detach().cpu().double().numpy() if hasattr(a, "detach") else a, np.float64)


def scores(logits, score):
    """(s [T,N,E], which logits are finite)."""
    x = _np(logits)
    ok = np.isfinite(x)
    x = np.where(ok, x, 0.0)
    if score == "sigmoid":
        with np.errstate(over="ignore"):
            s = 1.0 / (1.0 + np.exp(-x))
    else:
        top = np.where(ok, x, -np.inf).max(axis=2, keepdims=True)
        e = np.exp(np.where(ok, x, -np.inf) - np.where(np.isfinite(top), top, 0.0))
        s = e / np.maximum(e.sum(axis=2, keepdims=True), 1e-300)
    return np.where(ok, s, 0.0), ok


def choose(logits, select_bias, token_mask, k, C, score="softmax", groups=1, kept=1, top=1, renorm=True, scale=1.0):
    T, N, E = logits.shape
    s, ok = scores(logits, score)
    b = np.zeros((T, E)) if select_bias is None else _np(select_bias)
    on = ok & np.isfinite(b)[:, None, :]
    if token_mask is not None:
        on = on & (np.asarray(token_mask.cpu() if hasattr(token_mask, "cpu") else token_mask) != 0)[:, :, None]
    # without a bias the order is that of the logits
    value = np.where(on, s + np.where(np.isfinite(b), b, 0.0)[:, None, :], -np.inf)
    order_by = np.where(on, _np(logits), -np.inf) if select_bias is None else value
    idx = np.full((T, N, k), -1, np.int64)
    for t in range(T):
        for n in range(N):
            c = order_by[t, n].copy()
            if groups > 1:
                v = (order_by if select_bias is None and top == 1 else value)[t, n].reshape(groups, -1)
                g = np.sort(v, axis=1)[:, ::-1][:, :top].sum(axis=1)
                shut = np.ones(groups, bool)
                shut[np.argsort(-g, kind="stable")[:kept]] = False
                c.reshape(groups, -1)[shut] = -np.inf
            best = np.argsort(-c, kind="stable")[:k]
            best = best[np.isfinite(c[best])]
            idx[t, n, :len(best)] = best
    there = idx >= 0
    mine = np.where(there, np.take_along_axis(s, np.maximum(idx, 0), axis=2), 0.0)
    mass = mine.sum(axis=2, keepdims=True)
    share = mine / np.where(mass > 0, mass, 1.0) if renorm else mine
    slot = np.full((T, N, k), -1, np.int64)
    demand = np.zeros((T, E), np.int64)
    for t in range(T):
        for j in range(k):
            for n in range(N):
                e = idx[t, n, j]
                if e >= 0:
                    if demand[t, e] < C:
                        slot[t, n, j] = demand[t, e]
                    demand[t, e] += 1
    return dict(idx=idx, gate=scale * share, share=share, slot=slot, demand=demand, load=np.minimum(demand, C), s=s)


def choose_bwd(ref, logits, x, w_router, dy, ye, score="softmax", renorm=True, scale=1.0):
    """dgate, dlogits, dW_r, dbias and the router's share of dX of <dY, y>, choices and slots held fixed."""
    idx, slot, share, s = ref["idx"], ref["slot"], ref["share"], ref["s"]
    T, N, k = idx.shape
    E = s.shape[2]
    x, w, dy, ye = _np(x), _np(w_router), _np(dy), _np(ye)
    dgate = np.zeros((T, N, k))
    for t in range(T):
        for j in range(k):
            n = np.nonzero(slot[t, :, j] >= 0)[0]
            dgate[t, n, j] = (dy[t, n] * ye[t, idx[t, n, j], slot[t, n, j]]).sum(axis=1)
    mean = (share * dgate).sum(axis=2, keepdims=True)
    dl = np.zeros((T, N, E))
    if score == "softmax" and not renorm:
        dense = np.zeros((T, N, E))
        t, n, j = np.nonzero(idx >= 0)
        dense[t, n, idx[t, n, j]] = dgate[t, n, j]
        dl = np.where((idx >= 0).any(axis=2, keepdims=True), scale * s * (dense - mean), 0.0)
    else:
        t, n, j = np.nonzero(idx >= 0)
        c = scale * share * (dgate - mean if renorm else dgate)
        if score == "sigmoid":
            c = c * (1.0 - np.take_along_axis(s, np.maximum(idx, 0), axis=2))
        dl[t, n, idx[t, n, j]] = c[t, n, j]
    return dict(dgate=dgate, dlogits=dl, dw_router=np.einsum("tnd,tne->tde", x, dl), dbias=dl.sum(axis=1),
                dx=np.einsum("tne,tde->tnd", dl, w))
