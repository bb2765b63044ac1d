"""GPU parity of the optimizer steps over many tensors with their oracles in 64 bits.

Tolerances, from the arithmetic (u = 2^-24, half a step of fp32):
    sum of squares   fp64 products are exact, sums of n terms off by at most n 2^-53 of the (positive) result
    m                two products, a sum, the clipping product and 1 - beta1: 4 u (|beta1 m| + |(1 - beta1) g|)
    v                positive terms of at most five roundings each: 6 u v
    param            decay and the last sum 3 u |p|, update 12 u of itself, m's error through it
    8-bit moments    formed in fp64 on both sides: the same codes.  param as above with m and v rounded once
    bf16 copies      the rounding of the fp32 parameters that the step wrote, bit for bit"""
import numpy as np
import pytest
import torch

from oracle import adamw_oracle as A
from oracle import state8_oracle as S
from paper_2601_02609_amd import inputs as I

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SIZES = [1, 3, 7, 8, 9, 127, 128, 129, 255, 2047, 2048, 2049, 5000, 100003, 0, 2056]


@pytest.fixture(scope="module")
def B():
    from paper_2601_02609_amd import binding
    binding.lib()
    return binding


def _flat(sizes, dtype, fill=0):
    """Tensors in the middle of one buffer, 128 values apart at least, and a check of what lies between them."""
    starts = np.cumsum([128] + [(n + 127) // 128 * 128 + 128 for n in sizes])
    whole = torch.full((int(starts[-1]),), 7, dtype=dtype, device="cuda")
    views = [whole[a:a + n] for a, n in zip(starts, sizes)]
    for x in views:
        x.fill_(fill)
    gaps = torch.ones(len(whole), dtype=torch.bool, device="cuda")
    for a, n in zip(starts, sizes):
        gaps[a:a + n] = False
    return views, lambda: bool((whole[gaps] == 7).all())


class _Tensors:
    """Parameters, gradients and moments of a list of tensors, in the library's form and in the oracle's."""

    def __init__(self, B, sizes, state8, bf16, seed=0, copies=True):
        rng = np.random.default_rng(seed)
        self.sizes, self.state8, self.bf16 = sizes, state8, bf16
        self.p = [(rng.standard_normal(n) * 0.1).astype(np.float32) for n in sizes]
        pd, ok_p = _flat(sizes, torch.float32)
        pb, ok_b = _flat(sizes, torch.bfloat16)
        m32, ok_m = _flat(sizes, torch.float32)
        v32, ok_v = _flat(sizes, torch.float32)
        m8, ok_m8 = _flat(sizes, torch.uint8)
        v8, ok_v8 = _flat(sizes, torch.uint8)
        ms, ok_ms = _flat([(n + 127) // 128 for n in sizes], torch.uint8)
        vs, ok_vs = _flat([(n + 127) // 128 for n in sizes], torch.uint8)
        for d, p in zip(pd, self.p):
            d.copy_(torch.from_numpy(p))
        self.intact = lambda: all(f() for f in (ok_p, ok_b, ok_m, ok_v, ok_m8, ok_v8, ok_ms, ok_vs))
        self.pd, self.pb = pd, pb if copies else [None] * len(sizes)
        self.md = [m8[i] if e else m32[i] for i, e in enumerate(state8)]
        self.vd = [v8[i] if e else v32[i] for i, e in enumerate(state8)]
        self.ms, self.vs = ms, vs
        self.lr_scale = [16.0 if i % 3 == 1 else 1.0 for i in range(len(sizes))]
        self.wd = [0.0 if i % 4 == 2 else 0.1 for i in range(len(sizes))]
        self.rng = rng
        self.new_grads()
        self.list = B.OptimTensors(self.gd, self.pd, self.md, self.vd, params_bf16=self.pb, m_scales=ms, v_scales=vs,
                                   lr_scale=self.lr_scale, weight_decay=self.wd)

    def new_grads(self):
        self.g = [(self.rng.standard_normal(n) * np.exp(self.rng.uniform(-9, -2, n))).astype(np.float32) for n in self.sizes]
        self.g = [I.bf16_bits_to_f32(I.f32_to_bf16_bits(g)) if b else g for g, b in zip(self.g, self.bf16)]
        self.gd = [torch.from_numpy(g).cuda().to(torch.bfloat16 if b else torch.float32) for g, b in zip(self.g, self.bf16)]

    def host(self, i):
        return [x.cpu().numpy() for x in (self.pd[i], self.md[i], self.ms[i], self.vd[i], self.vs[i])]


def _check_step(T, before, clip, step, seed, hp):
    f32 = lambda x: float(np.float32(x))
    b1, b2, eps = f32(hp["beta1"]), f32(hp["beta2"]), f32(hp["eps"])
    for i, n in enumerate(T.sizes):
        if n == 0:
            continue
        p0, m0, ms0, v0, vs0 = before[i]
        p1, m1, ms1, v1, vs1 = T.host(i)
        lr, wd = float(np.float32(hp["lr"]) * np.float32(T.lr_scale[i])), f32(T.wd[i])
        if T.state8[i]:
            p, state, m, v = S.step(p0, T.g[i], (m0, ms0, v0, vs0), step, seed, lr, b1, b2, eps, wd, clip=clip)
            for name, got, want in zip(("m", "m scale", "v", "v scale"), (m1, ms1, v1, vs1), state):
                assert np.array_equal(got, want), (i, n, name, int((got != want).sum()))
            em = U * np.abs(m)
        else:
            p, m, v = A.adamw_step(p0, T.g[i], m0, v0, step, lr, b1, b2, eps, wd, clip=clip)
            em = 4 * U * (np.abs(b1 * m0) + np.abs((1 - b1) * clip * T.g[i].astype(np.float64)))
            assert np.all(np.abs(m1 - m) <= em + 1e-45), i
            assert np.all(np.abs(v1 - v) <= 6 * U * v + 1e-45), i
        den = np.sqrt(v / (1 - b2 ** step)) + eps
        update = lr * (m / (1 - b1 ** step)) / den
        tol = 3 * U * (np.abs(p0) + np.abs(p)) + 12 * U * np.abs(update) + lr * em / (1 - b1 ** step) / den
        assert np.all(np.abs(p1 - p) <= tol), (i, n, float((np.abs(p1 - p) / tol).max()))
        if T.pb[i] is not None:
            assert np.array_equal(T.pb[i].view(torch.int16).cpu().numpy().view(np.uint16), I.f32_to_bf16_bits(p1)), i


@pytest.mark.parametrize("state8", ["32", "8", "both"])
@pytest.mark.parametrize("grads", ["fp32", "bf16", "both"])
def test_steps_match_the_oracle(B, state8, grads):
    """Three steps from zero moments, each checked from the state that the one before left, over odd sizes."""
    sizes = SIZES + [130 + i for i in range(60)]                            # more than one launch holds
    flags = {"32": lambda i: 0, "fp32": lambda i: 0, "8": lambda i: 1, "bf16": lambda i: 1, "both": lambda i: (i // 2) % 2}
    T = _Tensors(B, sizes, [flags[state8](i) for i in range(len(sizes))], [flags[grads](i + 1) for i in range(len(sizes))], seed=11)
    hp = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8)
    for step in (1, 2, 3):
        before = [T.host(i) for i in range(len(sizes))]
        clip = 0.37 if step == 2 else 1.0
        cd = torch.tensor([clip], device="cuda") if step == 2 else None
        print(f"[adamw multi] {state8} {grads} step {step}", flush=True)
        B.cce_adamw_multi_step(T.list, step, clip_coef=cd, seed=99, **hp)
        torch.cuda.synchronize()
        _check_step(T, before, float(np.float32(clip)), step, 99, hp)
        T.new_grads()
        T.list.set_grads(T.gd)
    assert T.intact()


@pytest.mark.parametrize("state8", [0, 1])
def test_large_tensor_and_no_copy(B, state8):
    T = _Tensors(B, [896 * 1201 + 3, 5], [state8] * 2, [0, 1], seed=12, copies=False)
    hp = dict(lr=3e-4, beta1=0.9, beta2=0.999, eps=1e-8)
    before = [T.host(i) for i in range(2)]
    B.cce_adamw_multi_step(T.list, 1000, seed=3, **hp)
    _check_step(T, before, 1.0, 1000, 3, hp)
    assert T.intact()


@pytest.mark.parametrize("hp,step", [(dict(lr=1e-2, beta1=0.0, beta2=0.0, eps=1e-8), 3), (dict(lr=0.0, beta1=0.9, beta2=0.999, eps=1e-8), 1),
                                     (dict(lr=1e-3, beta1=0.99, beta2=0.9999, eps=1e-3), 100000), (dict(lr=1e-3, beta1=0.5, beta2=0.5, eps=0.0), 2)])
@pytest.mark.parametrize("state8", [0, 1])
def test_other_hyperparameters(B, hp, step, state8):
    T = _Tensors(B, [3000, 129], [state8] * 2, [0, 0], seed=16)
    for k in (step, step + 1):
        before = [T.host(i) for i in range(2)]
        B.cce_adamw_multi_step(T.list, k, seed=8, **hp)
        _check_step(T, before, 1.0, k, 8, hp)
        T.new_grads()
        T.list.set_grads(T.gd)


def test_zero_gradient_and_eps_with_8_bit_moments(B):
    """0 / max(0, 2^-126): the parameters decay and nothing else, the moments stay zero."""
    T = _Tensors(B, [500], [1], [0], seed=17)
    T.gd[0].zero_()
    B.cce_adamw_multi_step(T.list, 1, lr=1e-3, eps=0.0)
    decay = np.float32(1) - np.float32(1e-3) * np.float32(0.1)
    assert np.array_equal(T.pd[0].cpu().numpy(), T.p[0] * decay)
    assert not bool(T.md[0].any()) and not bool(T.vd[0].any()) and bool((T.ms[0] == 127).all())


def test_step_of_one_tensor_equals_the_single_step(B):
    """Within the two calls' roundings of cce_adamw_step on the same tensor."""
    n = 100001
    T = _Tensors(B, [n], [0], [0], seed=13)
    p, m, v = (torch.from_numpy(T.p[0]).cuda(), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"))
    hp = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8)
    T.list = B.OptimTensors(T.gd, T.pd, T.md, T.vd, weight_decay=0.1)
    B.cce_adamw_multi_step(T.list, 1, **hp)
    B.cce_adamw_step(p, T.gd[0], m, v, 1, weight_decay=0.1, **hp)
    assert float((T.md[0] - m).abs().max()) <= 8 * U * float(m.abs().max())
    assert float((T.vd[0] - v).abs().max()) <= 12 * U * float(v.abs().max())
    assert float((T.pd[0] - p).abs().max()) <= 6 * U * float(p.abs().max()) + 48 * U * 1e-3


def test_state8_values_without_a_code_and_extremes(B):
    """NaN and infinite gradients spoil their own value only; zeros, the smallest and the largest values keep a scale."""
    n = 640
    T = _Tensors(B, [n], [1], [0], seed=14)
    g = T.g[0].copy()
    g[3], g[7], g[9] = np.nan, np.inf, -np.inf
    g[128:256] = 0.0
    g[256:384] = np.float32(1e-38) * np.arange(1, 129)
    g[384:512] = np.float32(3e37)
    g[512:520] = np.float32(1e-45)
    T.g[0] = g
    T.gd[0].copy_(torch.from_numpy(g))
    hp = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8)
    before = T.host(0)
    B.cce_adamw_multi_step(T.list, 1, seed=5, **hp)
    p1, m1, ms1, v1, vs1 = T.host(0)
    _, state, _, _ = S.step(before[0], g, (before[1], before[2], before[3], before[4]), 1, 5, 1e-3, float(np.float32(0.9)),
                            float(np.float32(0.999)), float(np.float32(1e-8)), 0.1)
    bad = ~np.isfinite(g)
    for got, want in zip((m1, v1), (state[0], state[2])):
        assert np.array_equal(got, want)
    assert np.array_equal(ms1, state[1]) and np.array_equal(vs1, state[3])
    assert np.isnan(p1[bad]).all() and np.isfinite(p1[:384][~bad[:384]]).all()
    m = B.cce_adamw_state8_read(T.md[0], T.ms[0])
    assert np.array_equal(np.isnan(m.cpu().numpy()), bad)


@pytest.mark.parametrize("n", [1, 7, 8, 127, 128, 129, 2049, 100003])
def test_state8_read_is_what_the_codes_stand_for(B, n):
    rng = np.random.default_rng(n)
    codes = rng.integers(0, 256, n).astype(np.uint8)
    scales = rng.integers(87, 168, (n + 127) // 128).astype(np.uint8)
    c, s = torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()
    (out,), intact = _flat([n], torch.float32)
    B.cce_adamw_state8_read(c, s, out=out)
    assert np.array_equal(out.cpu().numpy(), S.decode(codes, scales, S.M).astype(np.float32), equal_nan=True) and intact()
    B.cce_adamw_state8_read(c, s, second=True, out=out)
    assert np.array_equal(out.cpu().numpy(), (S.decode(codes, scales, S.R) ** 2).astype(np.float32), equal_nan=True) and intact()


def test_places_beyond_32_bits(B):
    """A tensor of over 2^32 values: its last ones, whose random numbers and addresses take the upper word in."""
    n, tail = (1 << 32) + 300, 1000
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    m, v = torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    ms, vs = (torch.zeros((n + 127) // 128, dtype=torch.uint8, device="cuda") for _ in range(2))
    rng = np.random.default_rng(18)
    first = (n - tail) // 128 * 128
    gt = I.f32_to_bf16_bits((rng.standard_normal(n - first) * 1e-2).astype(np.float32))
    g[first:] = torch.from_numpy(gt.view(np.int16)).cuda().view(torch.bfloat16)
    T = B.OptimTensors([g], [p], [m], [v], m_scales=[ms], v_scales=[vs])
    s, _ = B.cce_grad_sumsq_multi(T)
    gf = I.bf16_bits_to_f32(gt).astype(np.float64)
    assert abs(float(s) / float((gf ** 2).sum()) - 1.0) <= 1e-12
    B.cce_adamw_multi_step(T, 2, lr=1e-3, beta2=0.99, seed=21)
    um, ur = S.dither(n - first, 21, 2, first=first)
    b1, b2 = float(np.float32(0.9)), float(np.float32(0.99))
    for codes, scales, want in ((m, ms, S.encode((1 - b1) * gf, um, S.M)), (v, vs, S.encode(np.sqrt((1 - b2) * gf * gf), ur, S.R))):
        assert np.array_equal(codes[first:].cpu().numpy(), want[0]) and np.array_equal(scales[first // 128:].cpu().numpy(), want[1])
        assert not bool(codes[:first].any())
    assert bool((p[first:] != 0).any()) and not bool(p[:first].any())


def test_seed_and_step_choose_the_random_numbers(B):
    def run(seed, step):
        T = _Tensors(B, [5000, 300], [1, 1], [0, 0], seed=15)
        B.cce_adamw_multi_step(T.list, step, lr=1e-3, seed=seed)
        return torch.cat([T.md[0], T.vd[0], T.md[1]])
    a = run(1, 4)
    assert torch.equal(a, run(1, 4)) and not torch.equal(a, run(2, 4)) and torch.equal(a, run(1 + (1 << 32), 4))


@pytest.mark.parametrize("sizes,bf16", [([1], 0), ([3, 0, 8, 2049], 0), (SIZES, 2), ([100 + i for i in range(400)], 2), ([3_000_001, 17], 1), ([0, 0], 0)])
def test_sumsq_multi_and_clip(B, sizes, bf16):
    rng = np.random.default_rng(len(sizes))
    g = [(rng.standard_normal(n) * 0.05).astype(np.float32) for n in sizes]
    kinds = [bf16 if bf16 < 2 else i % 2 for i in range(len(sizes))]
    g = [I.bf16_bits_to_f32(I.f32_to_bf16_bits(x)) if k else x for x, k in zip(g, kinds)]
    T = B.OptimTensors([torch.from_numpy(x).cuda().to(torch.bfloat16 if k else torch.float32) for x, k in zip(g, kinds)])
    want = float(sum((x.astype(np.longdouble) ** 2).sum() for x in g))
    tol = (sum(sizes) + 4) * 2.0 ** -53 * want
    s, none = B.cce_grad_sumsq_multi(T)
    assert none is None and abs(float(s) - want) <= tol
    again, _ = B.cce_grad_sumsq_multi(T)
    assert torch.equal(s, again)
    for max_norm in (0.5, 1e6):
        s2, c = B.cce_grad_sumsq_multi(T, s.clone(), True, max_norm=max_norm, eps_norm=1e-6)
        assert abs(float(s2) - 2 * want) <= 3 * tol
        ref = min(1.0, max_norm / (np.sqrt(2 * want) + float(np.float32(1e-6))))
        assert abs(float(c) - ref) <= 2 * U * ref
    single = B.cce_clip_coef(s2, 1e6)
    assert float(single) == float(c)


def test_sumsq_of_non_finite_gradients(B):
    g = torch.ones(5000, device="cuda")
    g[4321] = float("inf")
    s, c = B.cce_grad_sumsq_multi(B.OptimTensors([g]), max_norm=1.0)
    assert float(s) == float("inf") and float(c) == 0.0
    g[4321] = 1e30                                                          # whose square fp32 does not hold
    s, _ = B.cce_grad_sumsq_multi(B.OptimTensors([g]))
    assert abs(float(s) / 1e60 - 1.0) <= 1e-6


def test_list_refuses(B):
    def new(**change):
        f = lambda dtype=torch.float32, n=300: [torch.zeros(n, dtype=dtype, device="cuda"), torch.zeros(8, dtype=dtype, device="cuda")]
        a = dict(grads=f(), params=f(), m=f(), v=f()) | change
        return B.OptimTensors(a.pop("grads"), a.pop("params"), a.pop("m"), a.pop("v"), **a)
    new()
    z = lambda n, dtype=torch.float32: torch.zeros(n, dtype=dtype, device="cuda")
    for change in (dict(params=[z(300)]), dict(params=[z(300), z(9)]), dict(params=None), dict(m=[z(300, torch.float16), z(8, torch.float16)]),
                   dict(grads=[z(300, torch.float16), z(8)]), dict(v=[z(600)[::2], z(8)]), dict(m=[z(300, torch.uint8), z(8)]),
                   dict(m=[z(300, torch.uint8), z(8)], v=[z(300, torch.uint8), z(8)]), dict(params_bf16=[z(300), None]),
                   dict(weight_decay=[0.1]), dict(lr_scale=[1.0, 1.0, 1.0]), dict(params=[z(300), None])):
        with pytest.raises(ValueError):
            new(**change)
    whole = z(400)
    new(grads=[whole[:300], whole[292:300]])                                # gradients are only read
    for change in (dict(params=[whole[:300], whole[292:300]]), dict(params=[whole[:300], z(8)], m=[z(300), whole[100:108]]),
                   dict(grads=[whole[:300], z(8)], v=[z(300), whole[:8]])):
        with pytest.raises(ValueError, match="overlaps"):
            new(**change)
    T = new(params_bf16=[None, z(8, torch.bfloat16)])
    with pytest.raises(ValueError):
        T.set_grads([z(300)])
    with pytest.raises(ValueError):
        T.set_grads([z(300), z(9)])
    with pytest.raises(ValueError, match="overlaps"):                       # and the gradients stay those that were
        T.set_grads([T._keep["params"][0], z(8)])
    T.set_grads([z(300, torch.bfloat16), z(8)])
    B.cce_adamw_multi_step(T, 1, lr=1e-3)
    with pytest.raises(ValueError):
        B.cce_adamw_multi_step(B.OptimTensors([z(5)]), 1, lr=1e-3)
    with pytest.raises(ValueError):
        B.cce_grad_sumsq_multi(T, accumulate=True)
    with pytest.raises(ValueError):
        B.cce_grad_sumsq_multi(T, clip_coef=z(1))
    with pytest.raises(B.CCEError):
        B.cce_adamw_multi_step(T, 0, lr=1e-3)
    with pytest.raises(B.CCEError):                                         # rows that do not start at 16 bytes
        B.cce_grad_sumsq_multi(B.OptimTensors([z(9)[1:]]))


def test_replaced_gradients_stay_until_the_stream_has_read_them(B):
    """Gradients replaced, and the memory asked for again, while a step on the caller's stream waits behind other work."""
    n = 1 << 22
    g = torch.randn(n, device="cuda")
    state = lambda: [torch.zeros(n, device="cuda") for _ in range(3)]
    want, got = state(), state()
    B.cce_adamw_multi_step(B.OptimTensors([g], *([x] for x in want)), 1, lr=1e-3)
    T = B.OptimTensors([g.clone()], *([x] for x in got))
    big, s = torch.empty(1 << 28, device="cuda"), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(50):                                                 # 50 GB of writes in front of the step
            big.fill_(1.0)
    B.cce_adamw_multi_step(T, 1, lr=1e-3, stream=s)
    T.set_grads([torch.zeros(n, device="cuda")])
    junk = [torch.full((n,), 9.0, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, got)) and len(junk) == 4


@pytest.mark.parametrize("bf16", [0, 1])
def test_state8_values_beyond_the_largest_scale(B, bf16):
    """A coefficient above 1 and gradients near fp32's end: values that no scale holds get a NaN code and leave the others of
    their block, the next ones' bytes above all, what they are."""
    n = 700
    T = _Tensors(B, [n], [1], [bf16], seed=19)
    g = T.g[0].copy()
    g[[5, 130, 131, 132, 133, 511]] = np.float32(2.0 ** 127) * np.float32(1.5)
    g[600] = np.float32(-2.0 ** 127)
    T.g[0] = g
    T.gd[0].copy_(torch.from_numpy(g))
    clip = 1000.0
    before = T.host(0)
    B.cce_adamw_multi_step(T.list, 1, lr=1e-3, clip_coef=torch.tensor([clip], device="cuda"), seed=5)
    p1, m1, ms1, v1, vs1 = T.host(0)
    _, state, _, _ = S.step(before[0], g, (before[1], before[2], before[3], before[4]), 1, 5, 1e-3, float(np.float32(0.9)),
                            float(np.float32(0.999)), float(np.float32(1e-8)), 0.1, clip=clip)
    big = np.abs(g) >= 2.0 ** 127
    m, r = S.decode(m1, ms1, S.M), S.decode(v1, vs1, S.R)
    assert np.array_equal(ms1, state[1]) and np.array_equal(vs1, state[3]) and (ms1[[0, 1, 3, 4]] == 247).all()
    assert np.array_equal(np.isnan(m), big) and np.array_equal(np.isnan(r), big)
    assert np.array_equal(m1[~big], state[0][~big]) and np.array_equal(v1[~big], state[2][~big])
    assert np.isfinite(p1[~big]).all() and T.intact()


def test_state8_read_of_an_empty_tensor(B):
    """A list takes tensors without values: their moments are read back like the others'."""
    z = lambda *shape, dtype=torch.uint8: torch.zeros(*shape, dtype=dtype, device="cuda")
    for shape in ((0,), (3, 0)):
        for second in (False, True):
            out = B.cce_adamw_state8_read(z(*shape), z(0), second=second)
            assert out.shape == shape and out.dtype == torch.float32 and out.is_cuda
    given = z(0, dtype=torch.float32)
    assert B.cce_adamw_state8_read(z(0), z(0), out=given) is given
    with pytest.raises(ValueError):
        B.cce_adamw_state8_read(z(0), z(1))


@pytest.mark.parametrize("what", ["grads", "params", "m", "v", "params_bf16"])
def test_a_tensor_that_is_not_aligned_is_named(B, what):
    """A view into a bucket that does not begin at 16 bytes is refused when the list is used, by its name."""
    f = lambda dtype=torch.float32: [torch.zeros(n, dtype=dtype, device="cuda") for n in (300, 9, 17)]
    a = dict(grads=f(), params=f(), m=f(), v=f(), params_bf16=f(torch.bfloat16))
    a[what][1] = a[what][1].new_zeros(24)[3:12]
    T = B.OptimTensors(a["grads"], a["params"], a["m"], a["v"], params_bf16=a["params_bf16"])
    with pytest.raises(B.CCEError, match=rf"{what}\[1\]") as refused:
        B.cce_adamw_multi_step(T, 1, lr=1e-3)
    assert refused.value.code == -1 and not any(bool(x.any()) for x in a["params"])
    if what == "grads":
        with pytest.raises(B.CCEError, match=r"grads\[1\]"):
            B.cce_grad_sumsq_multi(T)
    else:
        assert float(B.cce_grad_sumsq_multi(T)[0]) == 0.0                   # which reads the gradients alone
    with pytest.raises(B.CCEError, match="multi_step: "):                   # another reason: no tensor is named
        B.cce_adamw_multi_step(B.OptimTensors(f(), f(), f(), f()), 0, lr=1e-3)


@pytest.mark.parametrize("state8", [0, 1])
@pytest.mark.parametrize("bf16", [0, 1])
def test_step_with_copies_that_the_caches_do_not_hold(B, state8, bf16):
    """192 MiB of bf16 copies and more: two steps, the second one from nonzero moments, checked at both ends of each tensor and
    in the middle as the steps of small tensors are; the copies, and in the first step the parameters, everywhere."""
    sizes = [100_650_003, 7001, 130, 8000]
    assert 2 * sum(sizes) >= 192 << 20
    hp, seed, clip = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8), 31, 0.37
    gen = torch.Generator(device="cuda").manual_seed(20)
    rand = lambda n, std: torch.randn(n, device="cuda", generator=gen).mul_(std)
    kind = torch.uint8 if state8 else torch.float32
    z = lambda of, dtype: [torch.zeros(of(n), dtype=dtype, device="cuda") for n in sizes]
    same, blocks = (lambda n: n), (lambda n: (n + 127) // 128)
    p, pb, m, v = [rand(n, 0.1) for n in sizes], z(same, torch.bfloat16), z(same, kind), z(same, kind)
    ms, vs = (z(blocks, torch.uint8), z(blocks, torch.uint8)) if state8 else (None, None)
    new_grads = lambda: [rand(n, 1e-3).to(torch.bfloat16 if bf16 else torch.float32) for n in sizes]
    g = new_grads()
    T = B.OptimTensors(g, p, m, v, params_bf16=pb, m_scales=ms, v_scales=vs, weight_decay=0.1)
    f32 = lambda x: float(np.float32(x))
    b1, b2, eps, lr, wd, clip = f32(hp["beta1"]), f32(hp["beta2"]), f32(hp["eps"]), f32(hp["lr"]), f32(0.1), f32(clip)
    parts = []
    for i, n in enumerate(sizes):
        for first in {0, n // 2 // 128 * 128, max(0, n - 1500) // 128 * 128}:
            parts.append((i, first, min(n, first + 2048)))                  # whole blocks, whose largest value fixes their scale
    host = lambda x, a, b: x[a:b].float().cpu().numpy() if x.dtype == torch.bfloat16 else x[a:b].cpu().numpy()
    cut = lambda i, a, b: ([host(x[i], a, b) for x in (p, m, v)], [host(x[i], a // 128, (b + 127) // 128) for x in (ms, vs)] if state8 else None)
    for step in (1, 2):
        before = [cut(*part) for part in parts]
        whole0 = p[0].clone()
        print(f"[adamw multi] state8={state8} bf16={bf16} step {step}", flush=True)
        B.cce_adamw_multi_step(T, step, clip_coef=torch.tensor([clip], device="cuda"), seed=seed, **hp)
        for (i, a, b), ((p0, m0, v0), scales0) in zip(parts, before):
            (p1, m1, v1), scales1 = cut(i, a, b)
            gp = host(g[i], a, b)
            if state8:
                want_p, _, want_m, want_v = S.step(p0, gp, (m0, scales0[0], v0, scales0[1]), step, seed, lr, b1, b2, eps, wd, clip=clip)
                um, ur = S.dither(b - a, seed, step, first=a)
                for got, got_s, want in ((m1, scales1[0], S.encode(want_m, um, S.M)), (v1, scales1[1], S.encode(np.sqrt(want_v), ur, S.R))):
                    assert np.array_equal(got[:b - a], want[0]) and np.array_equal(got_s, want[1]), (i, a)
                em = U * np.abs(want_m)
            else:
                want_p, want_m, want_v = A.adamw_step(p0, gp, m0, v0, step, lr, b1, b2, eps, wd, clip=clip)
                em = 4 * U * (np.abs(b1 * m0) + np.abs((1 - b1) * clip * gp.astype(np.float64)))
                assert np.all(np.abs(m1 - want_m) <= em + 1e-45) and np.all(np.abs(v1 - want_v) <= 6 * U * want_v + 1e-45), (i, a)
            den = np.sqrt(want_v / (1 - b2 ** step)) + eps
            update = lr * (want_m / (1 - b1 ** step)) / den
            tol = 3 * U * (np.abs(p0) + np.abs(want_p)) + 12 * U * np.abs(update) + lr * em / (1 - b1 ** step) / den
            assert np.all(np.abs(p1 - want_p) <= tol), (i, a)
        assert all(torch.equal(x.view(torch.int16), y.bfloat16().view(torch.int16)) for x, y in zip(pb, p))
        if step == 1:                                                       # from zero moments: the update is lr g / (|g| + eps)
            gd = g[0].double() * clip
            update = lr * gd / (gd.abs() + eps)
            want = whole0.double() * (1.0 - lr * wd) - update
            over = (p[0].double() - want).abs() - 3 * U * (whole0.double().abs() + want.abs()) - 16 * U * update.abs()
            assert float(over.max()) <= 0.0
            del gd, update, want, over
        g = new_grads()
        T.set_grads(g)
