"""fp64 CPU oracle for the embedding lookup and its gradient.

TEST INFRASTRUCTURE ONLY: the slow, plain definition the HIP kernels are checked against.  It shares no
code with the GPU path and imports nothing from the package.

    y_i   = scale * W[t_i]                             0 where t_i is ignore_index or outside [0, V)
    dW[v] = dW0[v] + scale * sum over {i : t_i = v} of dy_i
"""
from __future__ import annotations

import numpy as np

__all__ = ["takes_part", "forward", "backward"]


def takes_part(tokens, V: int, ignore_index: int):
    t = np.asarray(tokens, dtype=np.int64)
    return (t != ignore_index) & (t >= 0) & (t < V)


def forward(weight, tokens, ignore_index: int, scale: float = 1.0):
    """weight float64 [V, D]; float64 [N, D], not rounded."""
    out = np.zeros((len(tokens), weight.shape[1]))
    for i, ok in enumerate(takes_part(tokens, len(weight), ignore_index)):
        if ok:
            out[i] = scale * weight[tokens[i]]
    return out


def backward(d_out, tokens, V: int, ignore_index: int, scale: float = 1.0, dw0=None):
    """(dW, |dW0| + |scale| sum |dy|): the second is what rounding errors of any order of the sum are relative to."""
    dw = np.zeros((V, d_out.shape[1])) if dw0 is None else np.array(dw0, dtype=np.float64)
    size = np.abs(dw)
    for i, ok in enumerate(takes_part(tokens, V, ignore_index)):
        if ok:
            dw[tokens[i]] += scale * d_out[i]
            size[tokens[i]] += abs(scale) * np.abs(d_out[i])
    return dw, size
