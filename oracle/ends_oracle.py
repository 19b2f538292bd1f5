"""Plain forms, in 64 bits, of what stands before and behind the layer stack in
a training step: the embedding and its gradient, the norms and their adjoint,
the head's cross entropy and distillation with their gradients. Written from
the definitions.
"""
from __future__ import annotations

import numpy as np


def embed(tokens, table, scale=1.0):
    tokens = np.asarray(tokens)
    V = table.shape[0]
    out = np.zeros((*tokens.shape, table.shape[1]))
    ok = (tokens >= 0) & (tokens < V)
    out[ok] = table[tokens[ok]] * scale
    return out


def embed_grad(tokens, dy, V, scale=1.0, start=None):
    """(gradient, sum of the magnitudes of its terms, number of terms per class)"""
    d = dy.shape[-1]
    got, mag = np.zeros((V, d)), np.zeros((V, d))
    count = np.zeros(V, dtype=np.int64)
    for t, row in zip(np.asarray(tokens).ravel(), dy.reshape(-1, d)):
        if 0 <= t < V:
            got[t] += scale * row
            mag[t] += abs(scale) * np.abs(row)
            count[t] += 1
    if start is not None:
        got, mag = got + start, mag + np.abs(start)
    return got, mag, count


def norm(x, w, b=None, eps=1e-5, rms=False):
    m = 0.0 if rms else x.mean(-1, keepdims=True)
    xh = (x - m) / np.sqrt(((x - m) ** 2).mean(-1, keepdims=True) + eps)
    return xh * w + (0.0 if b is None else b)


def norm_grad(x, dy, w, eps=1e-5, rms=False, add=None):
    """dx, dw, db"""
    m = 0.0 if rms else x.mean(-1, keepdims=True)
    r = 1.0 / np.sqrt(((x - m) ** 2).mean(-1, keepdims=True) + eps)
    xh, g = (x - m) * r, dy * w
    mg = 0.0 if rms else g.mean(-1, keepdims=True)
    dx = r * (g - mg - xh * (g * xh).mean(-1, keepdims=True)) + (0.0 if add is None else add)
    return dx, (dy * xh).reshape(-1, x.shape[-1]).sum(0), dy.reshape(-1, x.shape[-1]).sum(0)


def teacher(top_classes, top_logits, V, temperature):
    """q [n, k] over the entries that count, 0 elsewhere; whether a row has any"""
    q = np.zeros(top_logits.shape)
    ok = (top_classes >= 0) & (top_classes < V) & ~(top_logits == -np.inf)
    for i in range(len(q)):
        if ok[i].any():
            v = top_logits[i][ok[i]] / temperature
            e = np.exp(v - v.max())
            q[i][ok[i]] = e / e.sum()
    return q, ok.any(1)


def head(h, w, classes, q, live, temperature=1.0, weight=None, grad_scale=1.0, mean=False):
    """A loss against lists of classes [n, k] with probabilities q: dict of loss, total, dh, dw, and the
    parts (z / T, lse, p, dz before the scale, scale, sum q log q) that bounds on rounding are made of."""
    n, V, T = h.shape[0], w.shape[0], temperature
    weight = np.ones(n) if weight is None else np.asarray(weight, dtype=np.float64)
    live = np.asarray(live) & (weight != 0)
    hz = np.where(live[:, None], h, 0.0)
    z = hz @ w.T / T
    top = z.max(1, keepdims=True)
    lse = top[:, 0] + np.log(np.exp(z - top).sum(1))
    p = np.exp(z - lse[:, None])
    loss, plogp = np.zeros(n), np.zeros(n)
    dz = np.zeros((n, V))
    for i in range(n):
        if not live[i]:
            continue
        dz[i] = p[i]
        for c, qq in zip(classes[i], q[i]):
            if qq > 0:
                loss[i] += qq * (np.log(qq) - (z[i, c] - lse[i]))
                plogp[i] += qq * np.log(qq)
                dz[i, c] -= qq
        dz[i] *= weight[i]
    loss *= T * T
    wsum = float((weight * live).sum())
    scale = grad_scale * T
    if mean:
        scale = scale / wsum if wsum else 0.0
    return {"loss": loss, "total": np.array([(weight * loss).sum(), wsum]), "dh": scale * (dz @ w),
            "dw": scale * (dz.T @ hz), "z": z, "lse": lse, "p": p, "dz": dz, "scale": scale, "live": live,
            "weight": weight, "temperature": T, "plogp": plogp}


def cross_entropy(h, w, targets, **kw):
    targets = np.asarray(targets)
    live = (targets >= 0) & (targets < w.shape[0])
    return head(h, w, np.where(live, targets, 0)[:, None], live[:, None].astype(float), live, **kw)


def distill(h, w, top_classes, top_logits, temperature=1.0, **kw):
    q, live = teacher(np.asarray(top_classes), np.asarray(top_logits, dtype=np.float64), w.shape[0], temperature)
    return head(h, w, top_classes, q, live, temperature=temperature, **kw)
