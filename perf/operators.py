"""The work that the embedding and optimizer operators are measured on, through the public binding.

A case is a dict of plain values.  "op" says which operator a pass goes through:

    lookup    cce_embedding_forward: rows of the bf16 [V, D] matrix, scaled
    grad      cce_embedding_backward: the lookup's gradient, into a new fp32 [V, D] or added to one
    norm      cce_grad_sumsq_multi: sum of squares of all gradients and the clipping coefficient
    adamw     cce_adamw_multi_step: moments in fp32
    adamw8    cce_adamw_multi_step: moments in 8 bits, and their values read back (cce_adamw_state8_read)

N tokens, D hidden size, V vocabulary; "ignore" is the fraction of positions that hold the ignore index
(padding), "zipf" the exponent of the token distribution (0: uniform), "scaled" whether rows are scaled by
sqrt(D).  For the optimizer, "layers" > 0 gives the tensors of a transformer of that many layers with hidden
size D, feed-forward size F and vocabulary V; layers = 0 gives "count" tensors of "total" values in all, their
odd sizes drawn from "sizes_seed".  "grads" is the gradients' type: "fp32", "bf16" or "mixed" in turn.

The tensors of an optimizer step lie in flat buffers, each at a multiple of 128 values; the gaps hold zeros.
With own = False, `run` is the plain form: elementary torch operations in fp32; in fp64 the sums of squares and the
moments that are rounded to 8 bits, where which way a value next to a border goes is part of the result.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

IGN = -100
DEV = "cuda"
BLOCK = 128                       # values that share a scale in 8-bit moments
NORM = dict(max_norm=1.0, eps_norm=1e-6)
ADAM = dict(lr=3e-4, beta1=0.9, beta2=0.999, eps=1e-8)
STEP, SEED = 17, 1234


def listed():
    return [
        # one decode step of one sequence: the first launch of the step, latency only
        dict(name="lookup_decode", op="lookup", N=1, D=896, V=151936, ignore=0.0, zipf=1.1, scaled=False),
        # the input of a training step of the largest configuration, rows scaled by sqrt(D)
        dict(name="lookup_7b", op="lookup", N=32768, D=3584, V=151936, ignore=0.05, zipf=1.1, scaled=True),
        # a ragged unit-test sized batch into a new gradient
        dict(name="grad_small", op="grad", N=257, D=64, V=1000, ignore=0.10, zipf=0.0, scaled=False, accumulate=False),
        # tied embeddings at the headline configuration: added to what the LM head's backward left in dW
        dict(name="grad_tied", op="grad", N=8192, D=896, V=151936, ignore=0.15, zipf=1.1, scaled=False, accumulate=True),
        # an untied embedding, small vocabulary, wide rows, a quarter padding: a new gradient
        dict(name="grad_untied", op="grad", N=16384, D=4096, V=32000, ignore=0.25, zipf=1.3, scaled=True, accumulate=False),
        # tied embeddings at the largest configuration
        dict(name="grad_tied_7b", op="grad", N=32768, D=3584, V=151936, ignore=0.05, zipf=1.1, scaled=True, accumulate=True),
        # the adapters and norms of a small fine-tuning run: many small tensors, few launches matter
        dict(name="norm_small", op="norm", layers=0, count=60, total=300007, sizes_seed=1, grads="fp32"),
        # all gradients of a 0.4 B model: the head's in fp32, the layers' in bf16 and fp32
        dict(name="norm_model", op="norm", layers=24, D=896, F=3584, V=151936, grads="mixed"),
        # the optimizer step of the small run
        dict(name="adamw_small", op="adamw", layers=0, count=60, total=300007, sizes_seed=1, grads="fp32"),
        # the optimizer step of the 0.4 B model
        dict(name="adamw_model", op="adamw", layers=24, D=896, F=3584, V=151936, grads="mixed"),
        # the same two with moments in 8 bits
        dict(name="adamw8_small", op="adamw8", layers=0, count=60, total=300007, sizes_seed=1, grads="fp32"),
        dict(name="adamw8_model", op="adamw8", layers=24, D=896, F=3584, V=151936, grads="bf16"),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["lookup", "grad", "grad", "norm", "adamw", "adamw8"])
    if op in ("lookup", "grad"):
        D = 8 * _log(rng, 1, 1024)
        N = min(_log(rng, 1, 65536), 32768 * 3584 // D)
        V = min(_log(rng, 2, 256000), 151936 * 3584 // D)
        case = dict(op=op, N=N, D=D, V=V, ignore=rng.choice([0.0, 0.05, 0.15, 0.4]),
                    zipf=rng.choice([0.0, 1.1, 1.3]), scaled=rng.random() < 0.5)
        if op == "grad":
            case["accumulate"] = rng.random() < 0.6
        return case
    count = _log(rng, 1, 300)
    return dict(op=op, layers=0, count=count, total=_log(rng, max(count, 1000), 300_000_000),
                sizes_seed=rng.randrange(1 << 30), grads=rng.choice(["fp32", "bf16", "mixed"]))


# ---------------------------------------------------------------- what a program has in hand

def _token_probabilities(case):
    p = np.arange(1, case["V"] + 1, dtype=np.float64) ** -case["zipf"]
    return p / p.sum()


def _sizes(case):
    if case["layers"]:
        D, F = case["D"], case["F"]
        layer = [D * D, D * D, D * D // 4, D * D // 4, D * F, D * F, F * D, D, D]
        return [case["V"] * D] + layer * case["layers"] + [D]
    rng = random.Random(case["sizes_seed"])
    share = [math.exp(rng.uniform(0.0, 6.0)) for _ in range(case["count"])]
    return [max(1, int(case["total"] * s / sum(share))) for s in share]


def _prepare_tokens(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    N, D, V = case["N"], case["D"], case["V"]
    cdf = torch.from_numpy(np.cumsum(_token_probabilities(case))).to(DEV)
    tokens = torch.searchsorted(cdf, torch.rand(N, device=DEV, dtype=torch.float64, generator=gen)).clamp_(max=V - 1)
    tokens[torch.rand(N, device=DEV, generator=gen) < case["ignore"]] = IGN
    scale = float(np.float32(math.sqrt(D))) if case["scaled"] else 1.0
    s = dict(op=case["op"], tokens=tokens.to(torch.int32), V=V, scale=scale)
    if case["op"] == "lookup":
        s["weight"] = (torch.randn(V, D, device=DEV, generator=gen) * (2.5 / math.sqrt(D))).bfloat16()
        return s
    s["d_out"] = (torch.randn(N, D, device=DEV, generator=gen) * 1e-3).bfloat16()
    s["accumulate"] = case["accumulate"]
    s["d_weight"] = torch.randn(V, D, device=DEV, generator=gen) * 1e-3 if case["accumulate"] else torch.empty(V, D, device=DEV)
    return s


def _prepare_tensors(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    sizes = _sizes(case)
    padded = [(n + BLOCK - 1) // BLOCK * BLOCK for n in sizes]
    starts = np.cumsum([0] + padded[:-1]).tolist()
    T = sum(padded)
    inside = torch.zeros(T + 1, dtype=torch.int8, device=DEV)              # 1 where a tensor has a value, 0 in a gap
    inside[torch.tensor(starts, device=DEV)] += 1
    ends = torch.tensor([a + n for a, n in zip(starts, sizes)], device=DEV)
    inside.index_add_(0, ends, torch.full_like(ends, -1, dtype=torch.int8))
    inside = torch.cumsum(inside[:T], 0, dtype=torch.int8)

    def values(std):
        return torch.randn(T, device=DEV, generator=gen).mul_(std).mul_(inside)

    s = dict(op=case["op"], sizes=sizes, starts=starts, padded=padded, T=T)
    kinds = {"fp32": [0] * len(sizes), "bf16": [1] * len(sizes), "mixed": [i % 2 for i in range(len(sizes))]}[case["grads"]]
    s["kinds"] = kinds
    g = values(1e-3)
    s["grad_bf16"] = g.bfloat16() if any(kinds) else None
    s["grad_fp32"] = g if not all(kinds) else None
    if case["op"] == "norm":
        return s
    s["weight_decay"] = [0.1 if n > 8192 else 0.0 for n in sizes]          # norms and biases do not decay
    s["lr_scale"] = [16.0 if i % 7 == 3 else 1.0 for i in range(len(sizes))]
    s["clip"] = torch.rand(1, device=DEV, generator=gen) * 0.5 + 0.5
    s["param"] = values(0.02)
    s["param_bf16"] = s["param"].bfloat16()
    m, r = values(3e-4), values(1e-3).abs_()
    if case["op"] == "adamw":
        s["m"], s["v"] = m, r.mul_(r)
        return s
    half = torch.full((1, 1), 1 << 16, device=DEV)                         # to nearest
    s["m_code"], s["m_scale"] = _encode(m.view(-1, BLOCK).double(), half, 3)
    s["v_code"], s["v_scale"] = _encode(r.view(-1, BLOCK).double(), half >> 1, 4)
    return s


def prepare(case, seed):
    return _prepare_tokens(case, seed) if case["op"] in ("lookup", "grad") else _prepare_tensors(case, seed)


# ---------------------------------------------------------------- plain forms

def _valid(s):
    t = s["tokens"]
    return (t != IGN) & (t >= 0) & (t < s["V"])


def _plain_lookup(s):
    ok = _valid(s)
    rows = s["weight"][torch.where(ok, s["tokens"], 0).long()].float() * s["scale"]
    return torch.where(ok[:, None], rows, 0.0).bfloat16()


def _plain_grad(s):
    ok = _valid(s)
    rows = torch.where(ok[:, None], s["d_out"].float() * s["scale"], 0.0)
    spread = torch.arange(len(ok), device=DEV) % s["V"]                    # where the zeros of ignored rows go does not matter
    total = s["d_weight"] if s["accumulate"] else s["d_weight"].zero_()
    return total.index_add_(0, torch.where(ok, s["tokens"].long(), spread), rows)


def _per_block(s, per_tensor, dtype):
    """[blocks, 1]: for each block of the flat buffers what its tensor has."""
    blocks = [n // BLOCK for n in s["padded"]]
    return torch.repeat_interleave(torch.tensor(per_tensor, dtype=dtype, device=DEV), torch.tensor(blocks, device=DEV),
                                   output_size=s["T"] // BLOCK)[:, None]


def _blocks(flat):
    return flat.view(-1, BLOCK)


def _gradient(s):
    """All gradients as one fp32 tensor of blocks."""
    if s["grad_bf16"] is None:
        return _blocks(s["grad_fp32"])
    if s["grad_fp32"] is None:
        return _blocks(s["grad_bf16"]).float()
    return torch.where(_per_block(s, s["kinds"], torch.bool), _blocks(s["grad_bf16"]).float(), _blocks(s["grad_fp32"]))


def _plain_norm(s):
    sumsq = _gradient(s).double().square().sum().reshape(1)
    return dict(sumsq=sumsq, clip=(NORM["max_norm"] / (sumsq.sqrt() + NORM["eps_norm"])).clamp(max=1.0).float())


def _f32(x):
    return float(np.float32(x))


def _plain_update(s, m, v):
    """One AdamW step on s["param"] in fp32: the new moments, unrounded, in the type of m and v."""
    f = np.float32
    b1, b2 = _f32(ADAM["beta1"]), _f32(ADAM["beta2"])
    rates = [f(ADAM["lr"]) * f(x) for x in s["lr_scale"]]
    lr = _per_block(s, [float(x) for x in rates], torch.float32)
    decay = _per_block(s, [float(f(1) - x * f(wd)) for x, wd in zip(rates, s["weight_decay"])], torch.float32)
    g = _gradient(s).to(m.dtype) * s["clip"].to(m.dtype)
    m = m * b1 + g * (1.0 - b1)
    v = v * b2 + (g * (1.0 - b2)) * g
    top = m.float() * _f32(1.0 / (1.0 - b1 ** STEP))
    under = (v.float() * _f32(1.0 / (1.0 - b2 ** STEP))).sqrt() + _f32(ADAM["eps"])
    param = _blocks(s["param"])
    param.copy_(param * decay - lr * (top / under))
    s["param_bf16"].copy_(s["param"])
    return m, v


def _plain_adamw(s):
    m, v = _plain_update(s, _blocks(s["m"]), _blocks(s["v"]))
    s["m"].copy_(m.view(-1))
    s["v"].copy_(v.view(-1))
    return dict(param=s["param"], param_bf16=s["param_bf16"], m=s["m"], v=s["v"])


LOW = 0xFFFFFFFF


def _mix(h):
    h = h ^ (h >> 16)
    h = (h * 2891336453) & LOW
    h = h ^ (h >> 15)
    h = (h * 29943829) & LOW
    return h ^ (h >> 16)


def _dither(s):
    """32 bits for each value: a hash of its place in its tensor, the seed and the step."""
    at = _blocks(torch.arange(s["T"], device=DEV)) - _per_block(s, s["starts"], torch.int64)
    return _mix((at + _mix((SEED + _mix(STEP)) & LOW)) & LOW)


def _encode(x, dither, bits):
    """Codes with 4 exponent and `bits` mantissa bits (a sign in front if bits = 3) of x, and a scale byte a block, rounded by
    `dither`, 20 - bits random bits.  In 64 bits: which way a value next to a border goes is part of the result."""
    top = 448.0 if bits == 3 else 480.0
    a = x.abs()
    fine = a.isfinite()
    amax = torch.where(fine, a, 0.0).amax(1, keepdim=True)
    mant, e = torch.frexp(amax)                                            # mant in [0.5, 1)
    e = torch.where(amax == 0, 0, (e - 9 + (mant > top / 512.0).int()).clamp(-100, 120))
    y = torch.ldexp(a, -e)
    low = y < 2.0 ** -6
    high = torch.where(low, y + 2.0 ** -6, y).view(torch.int64) >> 32      # of 52 mantissa bits 20: a code's and those the dither meets
    code = ((high + dither) >> (20 - bits)) - torch.where(low, 1017 << bits, 1016 << bits)
    if bits == 3:
        code = torch.where(fine, code, 0x7F) | torch.where(x < 0, 0x80, 0)
    else:
        code = torch.where(fine, torch.where(x > 0, code.clamp(min=1), code), 0xFF)
    return code.to(torch.uint8).view(-1), (e + 127).to(torch.uint8).view(-1)


def _decode(code, scale, bits):
    c = _blocks(code).int()
    mag = c & 0x7F if bits == 3 else c
    field, mant = mag >> bits, mag & ((1 << bits) - 1)
    x = torch.where(field == 0, mant, mant + (1 << bits)).double()
    x = torch.ldexp(x, field.clamp(min=1) - 7 - bits + scale.int()[:, None] - 127)
    x = torch.where(mag == (0x7F if bits == 3 else 0xFF), torch.nan, x)
    return torch.where(c > 0x7F, -x, x) if bits == 3 else x


def _plain_moments8(s):
    """In 64 bits."""
    return _decode(s["m_code"], s["m_scale"], 3), _decode(s["v_code"], s["v_scale"], 4).square()


def _plain_adamw8(s):
    m, v = _plain_update(s, *_plain_moments8(s))
    h = _dither(s)
    for name, x, dither, bits in (("m", m, h >> 15, 3), ("v", v.sqrt(), h & 0xFFFF, 4)):
        code, scale = _encode(x, dither, bits)
        s[name + "_code"].copy_(code)
        s[name + "_scale"].copy_(scale)
    m, v = _plain_moments8(s)
    return dict(param=s["param"], param_bf16=s["param_bf16"], m=m.float().view(-1), v=v.float().view(-1))


# ---------------------------------------------------------------- the framework's calls

def _cut(s, flat, per=1):
    """The tensors of a flat buffer that holds a value for every `per` values."""
    return None if flat is None else [flat[a // per:a // per + (n + per - 1) // per] for a, n in zip(s["starts"], s["sizes"])]


def _handle(B, s):
    """The list of tensors that a training program makes once and steps with."""
    if "handle" not in s:
        both = [_cut(s, s["grad_fp32"]), _cut(s, s["grad_bf16"])]
        grads = [both[k][i] for i, k in enumerate(s["kinds"])]
        if s["op"] == "norm":
            s["handle"] = B.OptimTensors(grads)
        else:
            eight = s["op"] == "adamw8"
            s["handle"] = B.OptimTensors(
                grads, _cut(s, s["param"]), _cut(s, s["m_code" if eight else "m"]), _cut(s, s["v_code" if eight else "v"]),
                params_bf16=_cut(s, s["param_bf16"]),
                m_scales=_cut(s, s["m_scale"], BLOCK) if eight else None,
                v_scales=_cut(s, s["v_scale"], BLOCK) if eight else None,
                lr_scale=s["lr_scale"], weight_decay=s["weight_decay"])
    return s["handle"]


def _run_own(s):
    from paper_2601_02609_amd import binding as B
    if s["op"] == "lookup":
        return B.cce_embedding_forward(s["tokens"], s["weight"], IGN, scale=s["scale"])
    if s["op"] == "grad":
        return B.cce_embedding_backward(s["tokens"], s["d_out"], s["V"], IGN, scale=s["scale"], d_weight=s["d_weight"],
                                        accumulate_dw=s["accumulate"])
    handle = _handle(B, s)
    if s["op"] == "norm":
        sumsq, clip = B.cce_grad_sumsq_multi(handle, **NORM)
        return dict(sumsq=sumsq, clip=clip)
    B.cce_adamw_multi_step(handle, STEP, clip_coef=s["clip"], seed=SEED, **ADAM)
    if s["op"] == "adamw":
        return dict(param=s["param"], param_bf16=s["param_bf16"], m=s["m"], v=s["v"])
    return dict(param=s["param"], param_bf16=s["param_bf16"], m=B.cce_adamw_state8_read(s["m_code"], s["m_scale"]),
                v=B.cce_adamw_state8_read(s["v_code"], s["v_scale"], second=True))


PLAIN = dict(lookup=_plain_lookup, grad=_plain_grad, norm=_plain_norm, adamw=_plain_adamw, adamw8=_plain_adamw8)


def run(state):
    return _run_own(state) if own else PLAIN[state["op"]](state)


# ---------------------------------------------------------------- floors

def work(case):
    if case["op"] in ("lookup", "grad"):
        N, D, V = case["N"], case["D"], case["V"]
        rows = N * (1.0 - case["ignore"])
        distinct = float((-np.expm1(rows * np.log1p(-np.minimum(_token_probabilities(case), 1 - 1e-12)))).sum())
        if case["op"] == "lookup":
            return dict(bytes=4.0 * N + 2.0 * D * (distinct + N), flops=rows * D)
        return dict(bytes=4.0 * N + 2.0 * D * rows + (8.0 * D * distinct if case["accumulate"] else 4.0 * V * D), flops=rows * D)
    sizes = _sizes(case)
    n = float(sum(sizes))
    grad = sum(size * (2.0 if case["grads"] == "bf16" or (case["grads"] == "mixed" and i % 2) else 4.0) for i, size in enumerate(sizes))
    if case["op"] == "norm":
        return dict(bytes=grad, flops=2.0 * n)
    if case["op"] == "adamw":
        return dict(bytes=grad + n * (12 + 12 + 2), flops=15.0 * n)
    blocks = sum((size + BLOCK - 1) // BLOCK for size in sizes)
    return dict(bytes=grad + n * (4 + 2 + 4 + 2 + 2) + 4.0 * blocks + n * 8, flops=15.0 * n)


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_tokens(case, s):
    t = s["tokens"].long()
    ok = (t >= 0) & (t < case["V"])
    if case["op"] == "lookup":
        out = torch.zeros(case["N"], case["D"], dtype=torch.float64, device=DEV)
        out[ok] = s["weight"][t[ok]].double() * s["scale"]
        return out
    out = s["d_weight"].double() if case["accumulate"] else torch.zeros(case["V"], case["D"], dtype=torch.float64, device=DEV)
    if bool(ok.any()):
        t, at = t[ok].sort(stable=True)
        sums = s["d_out"][ok][at].double().cumsum(0)                       # of sorted rows: a token's sum is a difference
        token, count = torch.unique_consecutive(t, return_counts=True)
        ends = sums[count.cumsum(0) - 1]
        out[token] += s["scale"] * torch.cat([ends[:1], ends[1:] - ends[:-1]])
    return out


def _exact_round(x, u, bits, top):
    """The values that x's codes stand for; u in [0, 1): the random part of a step."""
    x = x.reshape(-1, BLOCK)
    amax = x.abs().amax(1, keepdim=True)
    e = torch.ceil(torch.log2(amax / top)).clamp(-100, 120)
    e = torch.where(amax == 0, 0.0, e)
    y = x.abs() / torch.pow(2.0, e)
    step = torch.pow(2.0, torch.floor(torch.log2(y.clamp(min=2.0 ** -6))) - bits)
    q = torch.floor(y / step + u.reshape(-1, BLOCK)) * step
    if bits == 4:
        q = torch.where(y > 0, q.clamp(min=2.0 ** -10), q)
    return (torch.sign(x) * q * torch.pow(2.0, e)).reshape(-1)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("lookup", "grad"):
        return _exact_tokens(case, s)
    per = torch.tensor(s["padded"], device=DEV)
    g = s["grad_fp32"].double() if s["grad_fp32"] is not None else s["grad_bf16"].double()
    if case["grads"] == "mixed":
        for a, n, k in zip(s["starts"], s["padded"], s["kinds"]):
            if k:
                g[a:a + n] = s["grad_bf16"][a:a + n].double()
    if case["op"] == "norm":
        total = torch.dot(g, g).reshape(1)
        return dict(sumsq=total, clip=torch.clamp(NORM["max_norm"] / (total.sqrt() + NORM["eps_norm"]), max=1.0))
    f = {k: float(np.float32(v)) for k, v in ADAM.items()}
    rate = torch.repeat_interleave(torch.tensor(s["lr_scale"], dtype=torch.float64, device=DEV) * f["lr"], per)
    wd = torch.repeat_interleave(torch.tensor([float(np.float32(x)) for x in s["weight_decay"]], dtype=torch.float64, device=DEV), per)
    g *= s["clip"].double()
    if case["op"] == "adamw":
        m, v = s["m"].double(), s["v"].double()
    else:
        def values(code, scale, bits):                                     # every code's value, by the format's definition
            field, mant = [(c >> bits) & 15 for c in range(256)], [c & ((1 << bits) - 1) for c in range(256)]
            table = [(math.ldexp((1 << bits) + t, max(k, 1) - 7 - bits) if k else math.ldexp(t, -6 - bits)) for k, t in zip(field, mant)]
            if bits == 3:
                table = [-x if c > 127 else x for c, x in enumerate(table)]
            table = torch.tensor(table, dtype=torch.float64, device=DEV)
            return (table[code.long()].reshape(-1, BLOCK) * torch.pow(2.0, scale.double() - 127)[:, None]).reshape(-1)
        m = values(s["m_code"], s["m_scale"], 3)
        v = values(s["v_code"], s["v_scale"], 4) ** 2
    m = f["beta1"] * m + (1 - f["beta1"]) * g
    v = f["beta2"] * v + (1 - f["beta2"]) * g * g
    param = s["param"].double() * (1 - rate * wd)
    param -= rate * (m / (1 - f["beta1"] ** STEP)) / (torch.sqrt(v / (1 - f["beta2"] ** STEP)) + f["eps"])
    if case["op"] == "adamw8":
        h = _dither(s)                                                     # the random numbers are an input of the definition
        m = _exact_round(m, (h >> 15).double() / 2 ** 17, 3, 448.0)
        v = _exact_round(v.sqrt(), (h & 0xFFFF).double() / 2 ** 16, 4, 480.0) ** 2
    return dict(param=param, param_bf16=param, m=m, v=v)
