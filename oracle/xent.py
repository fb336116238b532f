"""The cross entropy of the LM head and its gradients in float64, from the definition:
cross entropy between the learnt distribution (1 - eps on the target, eps / V everywhere) and
softmax(h W^T), plus lambda lse^2, over the rows whose target lies in [0, V)."""

from __future__ import annotations

import numpy as np


def xent(h, w, target, eps=0.0, lam=0.0, reduction="mean"):
    """dict of loss, tok [T], n, dz [T, V] (of loss), mag [T, V] (the sum of the sizes of dz's
    terms), dh [T, d], dw [V, d], lse [T]. Rows without a label are zeros, whatever h holds."""
    h, w = np.asarray(h, np.float64), np.asarray(w, np.float64)
    T, V = h.shape[0], w.shape[0]
    target = np.asarray(target)
    rows = np.flatnonzero((target >= 0) & (target < V))
    n = len(rows)
    tok, lse = np.zeros(T), np.zeros(T)
    dz, mag = np.zeros((T, V)), np.zeros((T, V))
    z = h[rows] @ w.T
    m = z.max(1, keepdims=True, initial=-np.inf)
    e = np.exp(z - m)
    s = e.sum(1, keepdims=True)
    lse[rows] = (m + np.log(s))[:, 0]
    want = np.full((n, V), eps / V)
    want[np.arange(n), target[rows]] += 1.0 - eps
    tok[rows] = -(want * (z - m - np.log(s))).sum(1) + lam * lse[rows] ** 2
    weight = 1.0 if reduction == "sum" else 1.0 / max(n, 1)
    g = (1.0 + 2.0 * lam * lse[rows])[:, None]
    dz[rows] = weight * (g * e / s - want)
    mag[rows] = weight * (np.abs(g) * e / s + want)
    dh = np.zeros((T, h.shape[1]))
    dh[rows] = dz[rows] @ w
    return dict(loss=tok.sum() * weight, tok=tok, n=n, dz=dz, mag=mag, dh=dh, dw=dz[rows].T @ h[rows],
                lse=lse)
