"""fp64 CPU oracle for the router of a mixture-of-experts layer: top-k experts, their weights and counts, the balance and the z
loss, and the gradient of the logits.

TEST INFRASTRUCTURE ONLY: the slow, plain definition the HIP kernels are checked against.  It shares no code with the GPU path,
imports nothing from the package and is never called from the product path.  Rows are walked one by one, experts ranked by
sorting (value, -index) pairs.
"""
from __future__ import annotations

import numpy as np

__all__ = ["forward", "backward", "total"]


def forward(logits, top_k, taken=None, renormalize=True):
    """dict of indices, weights, lse, counts, prob_sums, losses, p; `taken`: bool [N], rows that take part (None: all)."""
    x = np.asarray(logits, dtype=np.float64)
    N, E = x.shape
    indices = np.full((N, top_k), -1, dtype=np.int32)
    weights = np.zeros((N, top_k))
    lse, p = np.zeros(N), np.zeros((N, E))
    n = 0
    for i in range(N):
        usable = [e for e in range(E) if not x[i, e] == -np.inf]
        if (taken is not None and not taken[i]) or not usable:
            continue
        n += 1
        order = sorted(usable, key=lambda e: (not np.isnan(x[i, e]), -x[i, e] if not np.isnan(x[i, e]) else 0.0, e))[:top_k]
        with np.errstate(invalid="ignore"):
            top = np.max(x[i, usable])
            ex = np.where(np.isneginf(x[i]), 0.0, np.exp(x[i] - top))
            p[i] = ex / ex.sum()
            lse[i] = top + np.log(ex.sum())
        w = p[i, order]
        indices[i, :len(order)] = order
        weights[i, :len(order)] = w / w.sum() if renormalize else w
    counts = np.bincount(indices[indices >= 0], minlength=E)
    m = max(n, 1)
    losses = np.array([E / (top_k * m * m) * (counts * p.sum(0)).sum(), (lse ** 2).sum() / m])
    return dict(indices=indices, weights=weights, lse=lse, counts=np.append(counts, n).astype(np.int32), prob_sums=p.sum(0), losses=losses, p=p)


def total(x, indices, counts, d_weights, d_losses, renormalize):
    """What `backward` differentiates, of one or more rows: <d_weights, weights> + d_losses . (balance, z), indices and counts held."""
    E, k, n = x.shape[1], indices.shape[1], max(int(counts[-1]), 1)
    value = 0.0
    for i in range(len(x)):
        chosen = indices[i] >= 0
        if not chosen.any():
            continue
        top = x[i].max()
        lse = top + np.log(np.exp(x[i] - top).sum())
        p = np.exp(x[i] - lse)
        w = np.where(chosen, p[np.maximum(indices[i], 0)], 0.0)
        if renormalize:
            w = w / w.sum()
        value += (d_weights[i] * w)[chosen].sum() + d_losses[0] * E / (k * n * n) * (counts[:E] * p).sum() + d_losses[1] * lse ** 2 / n
    return value


def backward(logits, indices, counts, d_weights, d_losses, renormalize=True):
    """Gradient of `total` in 64 bits, by the chain rule through the softmax's Jacobian."""
    x = np.asarray(logits, dtype=np.float64)
    N, E = x.shape
    k, n = indices.shape[1], max(int(counts[-1]), 1)
    out = np.zeros((N, E))
    for i in range(N):
        chosen = indices[i] >= 0
        if not chosen.any():
            continue
        top = x[i].max()
        lse = top + np.log(np.exp(x[i] - top).sum())
        p = np.exp(x[i] - lse)
        jacobian = np.diag(p) - np.outer(p, p)                            # d p_a / d x_b
        at = indices[i][chosen]
        dw = np.asarray(d_weights[i], dtype=np.float64)[chosen]
        if renormalize:
            s = p[at].sum()
            dw = np.linalg.solve(np.eye(len(at)) * s, dw - (dw * p[at]).sum() / s)
        d_p = d_losses[0] * E / (k * n * n) * counts[:E].astype(np.float64)
        np.add.at(d_p, at, dw)
        out[i] = jacobian @ d_p + d_losses[1] * 2.0 * lse / n * p
    return out
