"""CPU oracle for AdamW moments in 8 bits: the formats, their scales, the rounding and one step.

TEST INFRASTRUCTURE ONLY: the slow, plain definition the HIP kernels are checked against.  It shares no
code with the GPU path and imports nothing from the package.

A block of 128 values (the last one may be short) has a scale byte s, 2^(s - 127) the smallest power of two
between 2^-100 and 2^120 with which its largest finite magnitude is at most the format's largest value:

    first moment   E4M3: sign, 4 exponent bits (bias 7), 3 mantissa bits; 0x7f / 0xff NaN; at most 448
    second moment  its square root, without a sign: 4 exponent bits (bias 7), 4 mantissa bits; 0xff NaN; at most 480

A value between two codes goes up with the probability of its place between them: floor(place + u), u in
[0, 1) a multiple of 2^-17 (2^-16) taken from a hash.  A square root above 0 does not become 0.
"""
from __future__ import annotations

import numpy as np

__all__ = ["BLOCK", "M", "R", "decode", "encode", "dither", "step"]

BLOCK = 128
M, R = 3, 4                       # mantissa bits: first moment, square root of the second
LARGEST = {M: 448.0, R: 480.0}
NAN = {M: 0x7F, R: 0xFF}


def _code_values(bits: int):
    """What the codes without a sign stand for, by the definition of the format."""
    codes = np.arange(128 if bits == M else 256)
    field, mant = codes >> bits, (codes % (1 << bits)) / (1 << bits)
    values = np.where(field == 0, mant * 2.0 ** -6, (1.0 + mant) * 2.0 ** (field - 7.0))
    values[-1] = np.nan
    return values


def decode(codes, scales, bits: int):
    """float64 values of the codes (m, or sqrt(v))."""
    codes = np.asarray(codes, dtype=np.int64)
    table = _code_values(bits)
    table = np.concatenate([table, -table]) if bits == M else table
    return table[codes] * np.repeat(2.0 ** (np.asarray(scales, dtype=np.float64) - 127.0), BLOCK)[:len(codes)]


def encode(x, u, bits: int):
    """(codes, scales) of float64 x, rounded by u in [0, 1)."""
    x = np.asarray(x, dtype=np.float64)
    n = len(x)
    codes, scales = np.zeros(n, dtype=np.uint8), np.zeros((n + BLOCK - 1) // BLOCK, dtype=np.uint8)
    values = _code_values(bits)[:-1]
    for b in range(len(scales)):
        at = slice(b * BLOCK, min(n, (b + 1) * BLOCK))
        a = np.abs(x[at])
        fine = np.isfinite(a)
        top = a[fine].max() if fine.any() else 0.0
        e = -100 if top > 0.0 else 0
        while top > LARGEST[bits] * 2.0 ** e and e < 120:
            e += 1
        y = np.where(fine, a, 0.0) * 2.0 ** -e
        below = np.searchsorted(values, y, side="right") - 1               # the code at or below y
        above = values[np.minimum(below + 1, len(values) - 1)]
        gap = np.where(above > values[below], above - values[below], 1.0)
        code = below + (np.floor((y - values[below]) / gap + u[at]) >= 1.0)
        if bits == R:
            code = np.where((x[at] > 0.0) & (code == 0), 1, code)
        code = np.where(fine, code, NAN[bits])
        if bits == M:
            code = code + np.where(fine & np.signbit(x[at]), 128, 0)
        codes[at] = code
        scales[b] = e + 127
    return codes, scales


def _mix(h):
    h = np.asarray(h, dtype=np.uint64) & np.uint64(0xFFFFFFFF)
    h = h ^ (h >> np.uint64(16))
    h = (h * np.uint64(2891336453)) & np.uint64(0xFFFFFFFF)
    h = h ^ (h >> np.uint64(15))
    h = (h * np.uint64(29943829)) & np.uint64(0xFFFFFFFF)
    return h ^ (h >> np.uint64(16))


def dither(n: int, seed: int, t: int, first: int = 0):
    """(u for m, u for sqrt(v)) of the values first .. first + n - 1 of a tensor in step t."""
    key = _mix(np.uint64(seed) + _mix(np.uint64(t & 0xFFFFFFFF)))
    at = np.arange(first, first + n, dtype=np.uint64)
    h = _mix((at & np.uint64(0xFFFFFFFF)) + (at >> np.uint64(32)) * np.uint64(32310901) + key)
    return (h >> np.uint64(15)).astype(np.float64) / 2 ** 17, (h & np.uint64(0xFFFF)).astype(np.float64) / 2 ** 16


def step(p, g, state, t: int, seed: int, lr: float, beta1: float, beta2: float, eps: float, weight_decay: float,
         clip: float = 1.0):
    """One AdamW step: (new p, new state, unrounded m, unrounded v); state = (m codes, m scales, r codes, r scales)."""
    g = np.asarray(g, dtype=np.float64) * clip
    with np.errstate(invalid="ignore", over="ignore"):
        m = beta1 * decode(state[0], state[1], M) + (1.0 - beta1) * g
        v = beta2 * decode(state[2], state[3], R) ** 2 + (1.0 - beta2) * g * g
        p = np.asarray(p, dtype=np.float64) * (1.0 - lr * weight_decay)
        p = p - lr * (m / (1.0 - beta1 ** t)) / (np.sqrt(v / (1.0 - beta2 ** t)) + eps)
        um, ur = dither(len(g), seed, t)
        return p, (*encode(m, um, M), *encode(np.sqrt(v), ur, R)), m, v
