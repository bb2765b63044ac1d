"""fp64 CPU oracle for updates orthogonalised by Newton-Schulz products and for the Muon step around them.

TEST INFRASTRUCTURE ONLY: the slow, plain definition the HIP kernels are checked against.  It shares no code with the
GPU path, imports nothing from the package and is never called from the product path.

    X = G / (|G|_F + eps), transposed where G is taller than wide
    each step:  A = X X^T,  X = a X + (b A + c A A) X

`orthogonalize` is that in 64 bits.  `orthogonalize_rounded` rounds where the kernels may, and is otherwise the same: how far it is from
`orthogonalize` is how far the kernels may be, beside the order of their fp32 sums.

    h      X in fp16, the operand of the products
    l      what X has beyond h, a whole number of 2^-8 of h's last place
    A      its diagonal apart, the rest in fp16
    M      = b A + c A A the same; but in the steps behind which the product of the a is 8 or more the diagonal is in the fp16 operand, and
           only what that rounding leaves is apart, and what is beyond 60
    X      a (h + l) + M's diagonal (h + l) + the rest of M h

Of up to 64 rows all of M acts on X, with 22 bits of it; of up to 32 the rest of A and M have 22 bits too.
"""
from __future__ import annotations

import numpy as np

__all__ = ["orthogonalize", "orthogonalize_rounded", "muon_step"]


def _steps(coefficients, steps):
    c = np.asarray(coefficients, dtype=np.float32).astype(np.float64)
    return np.broadcast_to(c, (steps, 3))


def _start(g, eps):
    g = np.asarray(g, dtype=np.float64)
    x = g / (np.sqrt((g * g).sum()) + eps)
    return (x.T, True) if g.shape[0] > g.shape[1] else (x, False)


def orthogonalize(g, coefficients, steps, eps):
    x, tall = _start(g, eps)
    for a, b, c in _steps(coefficients, steps):
        gram = x @ x.T
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.T if tall else x


def _half(x, scale):
    return (x * scale).astype(np.float16).astype(np.float64) / scale


def _whole(x, scale):
    """In two 16-bit values."""
    h = _half(x, scale)
    return h + _half(x - h, scale)


def _apart(x, scale, rounded=_half):
    """A symmetric matrix as its diagonal and the rest, rounded."""
    diagonal = x.diagonal().copy()
    return diagonal, rounded(x - np.diag(diagonal), scale)


def _product(x, y):
    """Of two symmetric matrices held apart."""
    (dx, ox), (dy, oy) = x, y
    return np.diag(dx * dy) + dx[:, None] * oy + ox * dy[None, :] + ox @ oy


def _polynomial(gram, a, b, c):
    d, off = gram
    square = _product(gram, gram)
    return a * np.eye(len(d)) + b * (np.diag(d) + off) + c * square


def _rest(x, h):
    """x - h in eight bits below h's last place, h = fp16 of 2^13 x."""
    places = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(h) * 2.0 ** 13, 2.0 ** -14))) - 10 - 13)
    return np.clip(np.rint((x - h) / places * 256), -128, 127) / 256 * places


def orthogonalize_rounded(g, coefficients, steps, eps, pair=False):
    """pair: the first two steps are taken as one, with the next A from the first one's polynomial S as S (S A)."""
    x, tall = _start(g, eps)
    square = _whole if len(x) <= 32 else _half
    steps_left = list(_steps(coefficients, steps))
    while steps_left:
        h = square(x, 2.0 ** 13)
        gram = _apart(h @ h.T, 2.0 ** 13, square)
        a, b, c = steps_left.pop(0)
        keep, m = _apart(_polynomial(gram, a, b, c), 2.0 ** 10, square)
        if pair:
            pair = False
            gram = _apart(_product((keep, m), _apart(_product((keep, m), gram), 2.0 ** 13, square)), 2.0 ** 13, square)
            first, (a, b, c) = a, steps_left.pop(0)
            keep, m = _apart(_product(_apart(_polynomial(gram, a, b, c), 2.0 ** 10, square), (keep, m)), 2.0 ** 10, square)
            a = a * first
        if len(x) <= 64:
            x = keep[:, None] * x + m @ _whole(x, 2.0 ** 13)
            continue
        if np.prod([abs(later[0]) for later in steps_left]) >= 8.0:
            on_h = _half(np.clip(keep - a, -60.0, 60.0), 2.0 ** 10)
            keep, m = keep - on_h, m + np.diag(on_h)
        x = keep[:, None] * (h + _rest(x, h)) + m @ h
    return x.T if tall else x


def muon_step(p, g, momentum, coefficients, steps, eps, lr, mu, nesterov, weight_decay, clip=1.0, orthogonal=orthogonalize):
    """New (param, momentum) in 64 bits; lr is the matrix's own."""
    g = np.asarray(g, dtype=np.float64) * clip
    momentum = mu * np.asarray(momentum, dtype=np.float64) + (1.0 - mu) * g
    u = mu * momentum + (1.0 - mu) * g if nesterov else momentum
    return (1.0 - lr * weight_decay) * np.asarray(p, dtype=np.float64) - lr * orthogonal(u, coefficients, steps, eps), momentum
