"""Balance losses, block norms and AdamW in fp64 numpy, from their definitions, loop by loop where
that is the plainest form.  Test infrastructure, like the rest of the oracle."""
from __future__ import annotations

import numpy as np


def _np(a):
    return None if a is None else np.asarray(a.detach().double().cpu().numpy() if hasattr(a, "detach") else a, np.float64)


# ---------------------------------------------------------------------------------------------------
# Balance losses: logits [T,N,E], idx [T,N,k], mask [T,N] or None.


def balance(logits, idx, mask=None):
    """dict(count, tokens, excess, loss, prob [T,N,E], lse [T,N], on [T,N])."""
    x, idx = _np(logits), np.asarray(idx.cpu().numpy() if hasattr(idx, "cpu") else idx)
    T, N, E = x.shape
    k = idx.shape[2]
    on = np.ones((T, N), bool) if mask is None else np.asarray(mask.cpu().numpy() if hasattr(mask, "cpu") else mask) != 0
    on = on & ~np.all(np.isneginf(x), axis=2)
    prob, lse = np.zeros((T, N, E)), np.zeros((T, N))
    count, tokens = np.zeros((T, E), np.int64), on.sum(axis=1)
    for t in range(T):
        r = x[t][on[t]]
        top = r.max(axis=1, keepdims=True, initial=-np.inf)
        s = np.exp(r - top).sum(axis=1, keepdims=True)
        prob[t][on[t]] = np.exp(r - top) / s
        lse[t][on[t]] = (top + np.log(s))[:, 0]
        chosen = idx[t][on[t]].reshape(-1)
        chosen = chosen[(chosen >= 0) & (chosen < E)]
        count[t] = np.bincount(chosen, minlength=E)
    m = np.maximum(tokens, 1).astype(np.float64)
    importance = prob.sum(axis=1)
    excess = importance - tokens[:, None] / E
    loss = np.stack([E / (k * m * m) * (count * importance).sum(axis=1), E / (m * m) * (excess ** 2).sum(axis=1),
                     (lse ** 2).sum(axis=1) / m], axis=1)
    return dict(count=count, tokens=tokens, excess=excess, loss=loss, prob=prob, lse=lse, on=on, k=k)


def balance_bwd(fwd, dloss):
    """(dlogits, coefficient c [T,1,E], z lse [T,N,1]) for the weights dloss [T,3]."""
    dl, E = _np(dloss), fwd["count"].shape[1]
    m = np.maximum(fwd["tokens"], 1).astype(np.float64)
    c = dl[:, 0:1] * E / (fwd["k"] * m * m)[:, None] * fwd["count"] + dl[:, 1:2] * 2 * E / (m * m)[:, None] * fwd["excess"]
    c = c[:, None, :]
    z = (dl[:, 2] * 2 / m)[:, None, None] * fwd["lse"][:, :, None]
    p = fwd["prob"]
    return p * (c - (p * c).sum(axis=2, keepdims=True) + z), c, z


# ---------------------------------------------------------------------------------------------------
# Block norms: tokens [T,N,d], parameters [T,d] or None.


def norm_stats(v, rms, eps):
    mean = np.zeros(v.shape[:2] + (1,)) if rms else v.mean(axis=2, keepdims=True)
    return mean, 1.0 / np.sqrt(((v - mean) ** 2).mean(axis=2, keepdims=True) + eps)


def _par(a, none):
    return none if a is None else _np(a)[:, None, :]


def norm(v, w, b, rms, eps):
    mean, rstd = norm_stats(v, rms, eps)
    return (v - mean) * rstd * _par(w, 1.0) + _par(b, 0.0)


def block_z(x, y, post_w, post_b, gate, rho, rms, post, eps):
    y = _np(y)
    w = norm(y, post_w, post_b, rms, eps) if post else y
    return rho * _np(x) + _par(gate, 1.0) * w


def _norm_back(g, v, mean, rstd, rms):
    h = (v - mean) * rstd
    r = g - h * (g * h).mean(axis=2, keepdims=True)
    return rstd * (r if rms else r - g.mean(axis=2, keepdims=True))


def block_bwd(y, z, post_w, post_b, gate, pre_w, dz, du, rho, rms, post, eps):
    """Gradients, and for each parameter's gradient the sum of its terms' magnitudes (`mag`)."""
    y, z, dz, du = _np(y), _np(z), _np(dz), _np(du)
    ref = z if z is not None else y
    dzt = np.zeros_like(ref) if dz is None else dz.copy()
    out, mag = {}, {}
    if du is not None:
        mean, rstd = norm_stats(z, rms, eps)
        zh = (z - mean) * rstd
        dzt = dzt + _norm_back(du * _par(pre_w, 1.0), z, mean, rstd, rms)
        out["dpre_w"], mag["dpre_w"] = (du * zh).sum(axis=1), np.abs(du * zh).sum(axis=1)
        out["dpre_b"], mag["dpre_b"] = du.sum(axis=1), np.abs(du).sum(axis=1)
    if y is None:
        return dict(out, dx=dzt), mag
    out["dx"] = rho * dzt
    g = dzt * _par(gate, 1.0)
    w = yh = y
    if post:
        mean, rstd = norm_stats(y, rms, eps)
        yh = (y - mean) * rstd
        w = yh * _par(post_w, 1.0) + _par(post_b, 0.0)
        out["dpost_w"], mag["dpost_w"] = (g * yh).sum(axis=1), np.abs(g * yh).sum(axis=1)
        out["dpost_b"], mag["dpost_b"] = g.sum(axis=1), np.abs(g).sum(axis=1)
        out["dy"] = _norm_back(g * _par(post_w, 1.0), y, mean, rstd, rms)
    else:
        out["dy"] = g
    out["dgate"] = (dzt * w).sum(axis=1)
    mag["dgate"] = (np.abs(dzt) * (np.abs(yh * _par(post_w, 1.0)) + np.abs(_par(post_b, 0.0)))).sum(axis=1)
    return out, mag


# ---------------------------------------------------------------------------------------------------
# AdamW: flat arrays.


def mix(h):
    h = np.asarray(h, np.uint64) & np.uint64(0xffffffff)
    cut = lambda a: a & np.uint64(0xffffffff)  # noqa: E731
    h = cut((h ^ (h >> np.uint64(16))) * np.uint64(0x9e4a8af7))
    h = cut((h ^ (h >> np.uint64(15))) * np.uint64(0xa6bd2c99))
    return h ^ (h >> np.uint64(16))


def dither_bits(n, place, step, seed, first=0):
    """(low, high) 16-bit halves of the hashes of elements first .. first + n - 1."""
    i = np.arange(first, first + n, dtype=np.uint64) & np.uint64(0xffffffff)
    key = np.uint64((0x5e4087b3 * place + 0x339cd49b * step + 0xe32a5e87 * seed) & 0xffffffff)
    h = mix(i * np.uint64(0x51f6db5b) + key)
    return (h & np.uint64(0xffff)).astype(np.int64), (h >> np.uint64(16)).astype(np.int64)


def e4m3_encode(v, bits, root=False):
    """(values, scale of each 256, distance of the rounding from its border in steps, steps).  ``root``: v is
    sqrt(v), which does not become 0 where it is positive and its block has a scale, but one step at least."""
    n = v.size
    nb = (n + 255) // 256
    pad = np.zeros(nb * 256)
    pad[:n] = np.abs(v)
    scale = pad.reshape(nb, 256).max(axis=1) / 448
    scale[scale * 448 < 2.0 ** -100] = 0.0
    per = np.repeat(scale, 256)[:n]
    a = np.divide(np.abs(v), per, out=np.zeros(n), where=per > 0)
    grid = 2.0 ** (np.maximum(np.frexp(a)[1] - 1, -6) - 3)
    pos = a / grid + (16 * bits + 8) / 2.0 ** 20
    q = np.minimum(grid * np.floor(pos), 448)
    if root:
        q = np.where(a > 0, np.maximum(q, 2.0 ** -9), q)
    return np.copysign(q, v), scale, np.abs(pos - np.round(pos)), grid


def adamw(p, g, m, v, step, lr, beta1, beta2, eps, lr_scale=1.0, weight_decay=0.0, grad_scale=1.0):
    """(p, m, v, |update|)."""
    g = g * grad_scale
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    r = lr * lr_scale
    upd = r * (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return p * (1 - r * weight_decay) - upd, m, v, np.abs(upd)
