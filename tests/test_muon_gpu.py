"""GPU parity of the orthogonalising optimizer entry points with their oracle in 64 bits.

Tolerances.  The products' operands have 16 bits: how far that alone moves the result is what the oracle's rounded form says, r =
|rounded - exact| of the same matrix.  The kernels round at the same places or fewer; their fp32 sums (2^-24 a term) make
single values go the other way in a later rounding, which changes r by a part of itself: 1.5 r is allowed, and as r can be small by chance
where few rows are rounded, 2^-10 of the result over the square root of the smaller side (an operand's rounding is 2^-12 in the mean,
X is one four times in a step's A and M).  bf16 results are rounded once more, by 2^-8 of each value at most.  Single values: twice the rounded
form's largest error and the same share of the largest value.  (Multiples of the root mean square are no bound: of a 128 x 300
matrix of four directions the oracle's rounded form itself is 17.8 of them off, of others up to 26, as rows with much of the large directions
have most of the error.)  A parameter is off by lr times that,
and by fp32's rounding of the decay's factor, its product, the update's product and the sum: 4 * 2^-24 of |param| + |update|.
Momentum: two factors, two products, a sum and the clipping product, 5 * 2^-24 of the sum of magnitudes."""
import math

import numpy as np
import pytest
import torch

from oracle import muon_oracle as M

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
ABC = (3.4445, -4.7750, 2.0315)
EPS = 1e-7
SHAPES = [(1, 1), (1, 7), (9, 1), (3, 5), (16, 16), (17, 129), (64, 64), (63, 65), (65, 63), (128, 300), (300, 128), (127, 511), (129, 257),
          (192, 192), (256, 1024), (1024, 130), (16, 896), (896, 16), (33, 2049), (385, 641), (32, 2048), (2000, 29), (31, 2052), (64, 1024), (1000, 50), (128, 448), (448, 100), (449, 128),
          (97, 128), (65, 444), (2, 100), (16, 4096), (5000, 13), (17, 2305), (50, 1030), (2051, 33), (64, 16500)]


@pytest.fixture(scope="module")
def B():
    from paper_2601_02609_amd import binding
    binding.lib()
    return binding


def _matrix(m, n, seed, kind="noise", scale=1e-3):
    rng = np.random.default_rng(seed + 1000 * m + n)
    g = rng.standard_normal((m, n))
    if kind == "directions":
        g = 0.05 * g + rng.standard_normal((m, 4)) @ rng.standard_normal((4, n))
    elif kind == "rows":
        g *= np.exp(2.0 * rng.standard_normal((m, 1)))
    return (g * scale).astype(np.float32)


def _rounded(x, bf16):
    t = torch.from_numpy(np.ascontiguousarray(x))
    return (t.bfloat16().float() if bf16 else t).numpy()


def _check(got, g, steps=5, coefficients=ABC, eps=EPS, rate=1.0, bf16=True, extra=0.0, pair=False):
    """got: rate * orthogonalised g, or what is left of it after `extra` (absolute, by value)."""
    want = M.orthogonalize(g, coefficients, steps, eps)
    r = M.orthogonalize_rounded(g, coefficients, steps, eps, pair) - want
    chance = 2.0 ** -10 / math.sqrt(min(g.shape))
    off = 1.5 * np.linalg.norm(r) + chance * np.linalg.norm(want)
    most = 2.0 * np.abs(r).max() + chance * np.abs(want).max()
    d = np.abs(got - rate * want)
    own = rate * (2.0 ** -8 * np.abs(want) if bf16 else 0.0) + extra
    assert np.linalg.norm(d) <= rate * off + np.linalg.norm(own * np.ones_like(want)), (g.shape, np.linalg.norm(d) / (rate * np.linalg.norm(want)))
    assert (d <= rate * most + own).all(), (g.shape, ((d - own) / (rate * most)).max())


def _guarded(shapes, dtype, fill):
    """Matrices in one buffer, odd distances apart, and a check of what lies between them."""
    sizes = [m * n for m, n in shapes]
    starts = np.cumsum([5] + [s + 3 for s in sizes])
    whole = torch.full((int(starts[-1]) + 8,), fill, dtype=dtype, device="cuda")
    views = [whole[a:a + s].view(*shape) for a, s, shape in zip(starts, sizes, shapes)]
    gaps = torch.ones(len(whole), dtype=torch.bool, device="cuda")
    for a, s in zip(starts, sizes):
        gaps[a:a + s] = False
    return views, lambda: bool((whole[gaps] == fill).all())


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{s[0]}x{s[1]}")
def test_one_matrix(B, shape, bf16):
    for kind in ("noise", "directions"):
        g = _rounded(_matrix(*shape, 1, kind), bf16)
        x = torch.from_numpy(g).cuda()
        out, = B.cce_orthogonalize_multi([x.bfloat16() if bf16 else x])
        assert out.dtype == torch.bfloat16 and out.shape == x.shape
        _check(out.float().cpu().numpy().astype(np.float64), g)


@pytest.mark.parametrize("offset", [0, 1])
def test_many_matrices_and_nothing_beside_them(B, offset):
    shapes = SHAPES[offset::2] + [(0, 4), (5, 0)] + [(7, 70 + i) for i in range(60)]
    hosts = [_matrix(m, n, 2, "rows") for m, n in shapes]
    x, intact_x = _guarded(shapes, torch.float32, 7.0)
    for v, h in zip(x, hosts):
        v.copy_(torch.from_numpy(h))
    out, intact = _guarded(shapes, torch.bfloat16, 7.0)
    n = len(shapes)
    need = B.lib().cce_muon_workspace_bytes
    ws = torch.full((1 << 26,), 0xff, dtype=torch.uint8, device="cuda")            # NaN in every type
    got = B.cce_orthogonalize_multi(x, out, workspace=ws)
    assert got is out and intact() and intact_x() and need is not None and n > 48
    for v, h in zip(out, hosts):
        if h.size:
            _check(v.float().cpu().numpy().astype(np.float64), h)


@pytest.mark.parametrize("scale", [1e-38, 1e-20, 1e18, 1e36])
def test_scales_that_have_no_square_in_fp32(B, scale):
    for shape in ((40, 100), (200, 150), (24, 3000)):
        g = _matrix(*shape, 3, scale=scale)
        out, = B.cce_orthogonalize_multi([torch.from_numpy(g).cuda()], eps=0.0)
        _check(out.float().cpu().numpy().astype(np.float64), g, eps=0.0)


def test_zeros_and_values_that_are_not_finite(B):
    for shape in ((20, 30), (200, 130), (20, 2500)):
        x = [torch.from_numpy(_matrix(*shape, i)).cuda() for i in range(4)]
        x[0].zero_()
        x[1][3, 5] = math.inf
        x[2][-1, -1] = math.nan
        out = B.cce_orthogonalize_multi(x)
        assert bool((out[0] == 0).all()) and bool(out[1].isnan().all()) and bool(out[2].isnan().all())
        _check(out[3].float().cpu().numpy().astype(np.float64), _matrix(*shape, 3))
        assert bool(B.cce_orthogonalize_multi([x[0]], eps=0.0)[0].isnan().all())


@pytest.mark.parametrize("steps", [1, 2, 3, 6, 16])
def test_steps_and_coefficients(B, steps):
    rng = np.random.default_rng(steps)
    per = np.stack([rng.uniform(1.2, 3.5, steps), rng.uniform(-3.0, -0.5, steps), rng.uniform(0.1, 0.6, steps)], 1).astype(np.float32)
    per[:, 2] = np.minimum(per[:, 2], 1.0)
    for shape in ((30, 50), (150, 260), (2100, 20)):
        g = _matrix(*shape, 4)
        try:
            out, = B.cce_orthogonalize_multi([torch.from_numpy(g).cuda()], steps=steps, coefficients=per)
        except B.CCEError as error:                                               # beyond what 16 bits hold: refused, not wrong
            assert error.code == B.CCE_ERR_UNSUPPORTED
            continue
        _check(out.float().cpu().numpy().astype(np.float64), g, steps=steps, coefficients=per)
    g = _matrix(70, 90, 5)
    classic = np.broadcast_to(np.array([1.5, -0.5, 0.0], dtype=np.float32), (steps, 3))
    out, = B.cce_orthogonalize_multi([torch.from_numpy(g).cuda()], steps=steps, coefficients=classic)
    _check(out.float().cpu().numpy().astype(np.float64), g, steps=steps, coefficients=classic)


def _step_state(shapes, bf16, copies=True, seed=0):
    rng = np.random.default_rng(seed)
    g = [_rounded(_matrix(m, n, seed), bf16[i]) for i, (m, n) in enumerate(shapes)]
    p = [(rng.standard_normal(s) * 0.02).astype(np.float32) for s in shapes]
    mom = [_matrix(m, n, seed + 7, "directions", 2e-4) for m, n in shapes]
    dev = [torch.from_numpy(x).cuda() for x in g]
    dev = [x.bfloat16() if b else x for x, b in zip(dev, bf16)]
    return g, p, mom, dev, [torch.from_numpy(x).cuda() for x in p], [torch.from_numpy(x).cuda() for x in mom], \
        [torch.empty(s, dtype=torch.bfloat16, device="cuda") if copies else None for s in shapes]


def _check_step(state, after, lr, mu, nesterov, lr_scale, wd, clip, pair=False):
    g, p, mom, *_ = state
    pd, md, cd = after
    lr, mu, clip = (float(np.float32(x)) for x in (lr, mu, clip))
    for i in range(len(g)):
        rate = float(np.float32(lr) * np.float32(lr_scale[i]))
        want_p, want_m = M.muon_step(p[i], g[i], mom[i], ABC, 5, EPS, rate, mu, nesterov, float(np.float32(wd[i])), clip)
        got_m = md[i].cpu().numpy().astype(np.float64)
        assert (np.abs(got_m - want_m) <= 5 * U * (mu * np.abs(mom[i]) + np.abs(clip * g[i]))).all()
        # the direction as the kernels see it: from the stored momentum
        u = mu * got_m + (1 - mu) * clip * g[i].astype(np.float64) if nesterov else got_m
        kept = (1.0 - rate * float(np.float32(wd[i]))) * p[i].astype(np.float64)
        got_p = pd[i].cpu().numpy().astype(np.float64)
        extra = 4 * U * (np.abs(kept) + rate * np.abs(M.orthogonalize(u, ABC, 5, EPS)))
        _check(kept - got_p, u, rate=rate, bf16=False, extra=extra, pair=pair)
        if cd[i] is not None:
            assert torch.equal(cd[i], pd[i].bfloat16())
        assert np.isfinite(want_p).all()


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("copies", [True, False])
def test_muon_step(B, nesterov, copies):
    shapes = SHAPES + [(0, 3), (48, 4096)]
    bf16 = [i % 2 == 1 for i in range(len(shapes))]
    lr_scale = [0.2 * math.sqrt(max(max(s), 1)) for s in shapes]
    wd = [0.1 if i % 3 else 0.0 for i in range(len(shapes))]
    state = _step_state(shapes, bf16, copies)
    _, _, _, gd, pd, md, cd = state
    clip = torch.tensor([0.37], device="cuda")
    handle = B.MuonTensors(gd, pd, md, params_bf16=cd if copies else None, lr_scale=lr_scale, weight_decay=wd)
    B.cce_muon_multi_step(handle, lr=0.02, momentum=0.9, nesterov=nesterov, clip_coef=clip)
    keep = [i for i, s in enumerate(shapes) if s[0]]
    pick = lambda x: [x[i] for i in keep]  # noqa: E731
    _check_step([pick(x) for x in state], [pick(x) for x in (pd, md, cd)], 0.02, 0.9, nesterov, pick(lr_scale), pick(wd), 0.37)


def test_a_step_repeated_gives_the_same_bits(B):
    shapes = [(256, 700), (40, 60), (513, 129), (40, 3000), (600, 1800)]
    runs = []
    for _ in range(2):
        _, _, _, gd, pd, md, cd = _step_state(shapes, [False, True, False, True, False])
        handle = B.MuonTensors(gd, pd, md, params_bf16=cd)
        for _ in range(3):
            B.cce_muon_multi_step(handle, lr=0.01)
        runs.append([x.clone() for x in pd + md + cd])
    assert all(torch.equal(x, y) for x, y in zip(*runs))


def test_captured_step_replayed(B):
    shapes = [(256, 700), (40, 60), (700, 129), (16, 500), (2200, 16), (512, 1300)]
    _, _, _, gd, pd, md, cd = _step_state(shapes, [False, True, False, True, True, False])
    start = [x.clone() for x in pd + md]
    handle = B.MuonTensors(gd, pd, md, params_bf16=cd)
    ws = torch.empty(B.muon_workspace_bytes(handle), dtype=torch.uint8, device="cuda")
    want = []
    for _ in range(3):
        B.cce_muon_multi_step(handle, lr=0.01, workspace=ws)
        want.append([x.clone() for x in pd + md + cd])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.cce_muon_multi_step(handle, lr=0.01, workspace=ws)
    for x, s in zip(pd + md, start):
        x.copy_(s)
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(pd + md + cd, want[k])), k
        ws.fill_(0xff)                                                            # other work between replays


def test_on_a_stream_of_the_callers(B):
    side = torch.cuda.Stream()
    g = _matrix(200, 300, 9)
    x = torch.from_numpy(g).cuda()
    side.wait_stream(torch.cuda.current_stream())
    out, = B.cce_orthogonalize_multi([x], stream=side)
    shapes = [(100, 200), (30, 20)]
    state = _step_state(shapes, [False, False])
    _, _, _, gd, pd, md, cd = state
    handle = B.MuonTensors(gd, pd, md, params_bf16=cd)
    side.wait_stream(torch.cuda.current_stream())
    B.cce_muon_multi_step(handle, lr=0.01, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    _check(out.float().cpu().numpy().astype(np.float64), g)
    _check_step(state, (pd, md, cd), 0.01, 0.95, True, [1.0, 1.0], [0.0, 0.0], 1.0)


@pytest.mark.parametrize("shape", [(1, 1), (5, 7), (16, 16), (300, 13), (16, 512), (513, 3), (32, 769), (3000, 20), (60, 1100), (64, 5000)],
                         ids=lambda s: f"{s[0]}x{s[1]}")
def test_few_rows_are_off_by_their_last_rounding(B, shape):
    """X = Q G with Q from 64 bits, its 2-norm at most 3.4445^5 < 486: a result is off by bf16's half step and by the rounding to fp32 of Q, of G's
    scaled value, of r products and of r sums, (r + 3) 2^-24 of |row of Q| |column of X| <= 486 |column of X|."""
    for kind in ("noise", "directions", "rows"):
        g = _matrix(*shape, 13, kind)
        out, = B.cce_orthogonalize_multi([torch.from_numpy(g).cuda()])
        want = M.orthogonalize(g, ABC, 5, EPS)
        x = g.astype(np.float64) / (np.linalg.norm(g.astype(np.float64)) + EPS)
        column = np.linalg.norm(x, axis=0 if shape[0] <= shape[1] else 1, keepdims=True)
        off = np.abs(out.float().cpu().numpy().astype(np.float64) - want)
        assert (off <= 2.0 ** -8 * np.abs(want) + (1 + 2.0 ** -8) * (min(shape) + 3) * U * 486.0 * column).all()


PAIRED = [(512, 1280), (1400, 500), (513, 2000)]         # the first two steps are taken as one


@pytest.mark.parametrize("kind", ["noise", "directions", "rows"])
@pytest.mark.parametrize("shape", PAIRED, ids=lambda s: f"{s[0]}x{s[1]}")
def test_two_steps_taken_as_one(B, shape, kind):
    g = _matrix(*shape, 11, kind)
    x = torch.from_numpy(g).cuda()
    # S of the last two has values up to 8 and 7.8: their product is beyond the operands' range, so that these are taken one by one
    wide = np.array([[8.0, -32.0, 25.6], [7.78, -12.16, 3.8]], dtype=np.float32)
    for steps, coefficients, pair in ((5, ABC, True), (2, ABC, True), (3, np.array([ABC, (2.0, -1.5, 0.5), (1.875, -1.25, 0.375)]), True), (2, wide, False), (1, ABC, False)):
        out, = B.cce_orthogonalize_multi([x], steps=steps, coefficients=coefficients)
        _check(out.float().cpu().numpy().astype(np.float64), g, steps=steps, coefficients=coefficients, pair=pair)


def test_muon_step_of_two_steps_taken_as_one(B):
    state = _step_state(PAIRED, [True, False, True])
    _, _, _, gd, pd, md, cd = state
    handle = B.MuonTensors(gd, pd, md, params_bf16=cd, weight_decay=0.1)
    B.cce_muon_multi_step(handle, lr=0.02, momentum=0.9)
    _check_step(state, (pd, md, cd), 0.02, 0.9, True, [1.0] * 3, [0.1] * 3, 1.0, pair=True)


def test_matrices_of_every_form_in_a_list(B):
    """Small, thin, tiled, of two steps taken as one, and empty ones in turn: each as alone."""
    shapes = [(40, 60), (16, 3000), (300, 400), (512, 1400), (0, 5), (2500, 600), (70, 900), (33, 2200), (1, 1)]
    x = [torch.from_numpy(_matrix(m, n, 3)).cuda() for m, n in shapes]
    for o, v in zip(B.cce_orthogonalize_multi(x), x):
        if v.numel():
            assert torch.equal(o, B.cce_orthogonalize_multi([v])[0])


def test_thin_matrices_of_several_launches(B):
    """More than share their launches; each as alone, also with more columns than 64 workgroups sum in 256 each."""
    x = [torch.from_numpy(_matrix(16 + i % 5, 2100 + 10 * i, i)).cuda() for i in range(58)] + [torch.from_numpy(_matrix(40000, 9, 1)).cuda()]
    out = B.cce_orthogonalize_multi(x)
    for i in (0, 4, 55, 56, 57, 58):
        assert torch.equal(out[i], B.cce_orthogonalize_multi([x[i]])[0])
        _check(out[i].float().cpu().numpy().astype(np.float64), x[i].cpu().numpy())


def test_groups_share_a_workspace(B):
    """More matrices than a launch holds, and more workspace than a group may have."""
    shapes = [(512, 640)] * 250 + [(12000, 10000)] * 4
    x = [torch.from_numpy(_matrix(m, n, 20 + i)).cuda() for i, (m, n) in enumerate(shapes[:250])]
    gen = torch.Generator(device="cuda").manual_seed(1)
    x += [torch.randn(m, n, device="cuda", generator=gen) for m, n in shapes[250:]]
    table = B.MuonTensors(x, [torch.empty_like(t) for t in x], [torch.empty_like(t) for t in x])
    assert 0 < B.muon_workspace_bytes(table) <= 3 << 30
    out = B.cce_orthogonalize_multi(x)
    for i in (0, 55, 56, 239, 240, 249):
        _check(out[i].float().cpu().numpy().astype(np.float64), x[i].cpu().numpy())
    for o, t in zip(out[250:], x[250:]):
        y = t.double() / torch.linalg.norm(t.double())
        for _ in range(5):
            gram = y.T @ y
            y = ABC[0] * y + y @ (ABC[1] * gram + ABC[2] * (gram @ gram))
        # 2^-9 of the operands' rounding and at most 2^-8 of bf16's
        assert float(torch.linalg.norm(o.double() - y) / torch.linalg.norm(y)) <= 2.0 ** -9 + 2.0 ** -8


@pytest.mark.parametrize("shape,count", [((100, 4096), 3), ((6000, 300), 1), ((1024, 4096), 1), ((5001, 1030), 1), ((1090, 1100), 30), ((2048, 2048), 13), ((3583, 2100), 6), ((3590, 3600), 1), ((4096, 4096), 2)],
                         ids=lambda s: "x".join(map(str, s)) if isinstance(s, tuple) else str(s))
def test_large_matrices(B, shape, count):
    """Tiles of 256 x 256, split ones among them.  Values of one size: every 64 x 64 block is off by no more than the whole may be, twice."""
    gen = torch.Generator(device="cuda").manual_seed(shape[0] + count)
    x = [torch.randn(shape, device="cuda", generator=gen) for _ in range(count)]
    out = B.cce_orthogonalize_multi(x)
    for i in {0, count // 2, count - 1}:
        y = x[i].double() / (torch.linalg.norm(x[i].double()) + EPS)
        y = y if shape[0] <= shape[1] else y.T.contiguous()
        for _ in range(5):
            gram = y @ y.T
            y = ABC[0] * y + (ABC[1] * gram + ABC[2] * (gram @ gram)) @ y
        y = y if shape[0] <= shape[1] else y.T.contiguous()
        off = out[i].double() - y
        allowed = 2.0 ** -9 + 2.0 ** -8                                           # of the operands' rounding and of bf16's
        assert float(torch.linalg.norm(off)) <= allowed * float(torch.linalg.norm(y))
        pad = (0, -shape[1] % 64, 0, -shape[0] % 64)
        blocks = [torch.nn.functional.pad(t.square(), pad).unflatten(0, (-1, 64)).unflatten(2, (-1, 64)).sum((1, 3)) for t in (off, y)]
        assert bool((blocks[0].sqrt() <= 2 * allowed * blocks[1].sqrt()).all())
    if count > 1:
        assert torch.equal(out[1], B.cce_orthogonalize_multi(x)[1])


@pytest.mark.parametrize("rows,cols", [(16384, 65536), (1 << 24, 64)])
def test_the_most_values_a_matrix_may_have(B, rows, cols):
    """2^30.  Two rows of X each share a column and have nothing in common with the others, so that the result is made of 2 x 2 blocks, all alike."""
    half = min(rows, cols) // 2
    step = max(rows, cols) // (2 * half)
    g = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    x = g if rows <= cols else g.t()
    i = torch.arange(half, device="cuda")
    p, q = (i * 7919 % half) * step + step // 2, half * step + (i * 104729 % half) * step + step - 1
    x[i, p], x[half + i, p], x[half + i, q] = 1.0, 0.5, 1.0
    u, s, v = np.linalg.svd(np.array([[1.0, 0.0], [0.5, 1.0]]))
    s = s / math.sqrt(half * 2.25)
    for _ in range(5):
        s = ABC[0] * s + ABC[1] * s ** 3 + ABC[2] * s ** 5
    want = (u * s) @ v
    out, = B.cce_orthogonalize_multi([g], eps=0.0)
    y = out if rows <= cols else out.t()
    for row, col, value in ((i, p, want[0, 0]), (i, q, want[0, 1]), (half + i, p, want[1, 0]), (half + i, q, want[1, 1])):
        # 2^-9 of the operands' rounding, of a block's norm, and bf16's half step
        assert float((y[row, col].double() - value).abs().max()) <= 2.0 ** -9 * np.linalg.norm(want) + 2.0 ** -8 * abs(value)
        y[row, col] = 0.0
    assert int(torch.count_nonzero(out)) == 0


def test_refusals(B):
    x = torch.randn(4, 6, device="cuda")
    for bad in ([], [x.half()], [x.t()], [x[0]], [x.cpu()]):
        with pytest.raises((ValueError, IndexError)):
            B.cce_orthogonalize_multi(bad)
    with pytest.raises(ValueError):
        B.cce_orthogonalize_multi([x], [x.bfloat16(), x.bfloat16()])
    with pytest.raises(ValueError):
        B.cce_orthogonalize_multi([x], [torch.empty(6, 4, dtype=torch.bfloat16, device="cuda")])
    y = x.bfloat16()
    with pytest.raises(ValueError):
        B.cce_orthogonalize_multi([y], [y])
    for steps in (0, 17):
        with pytest.raises(B.CCEError):
            B.cce_orthogonalize_multi([x], steps=steps, coefficients=np.full((steps, 3), 0.5, dtype=np.float32))
    for c, code in (((8.0, 1.0, 1.0), B.CCE_ERR_UNSUPPORTED), ((3.0, -70.0, 0.0), B.CCE_ERR_UNSUPPORTED), ((math.nan, 0.0, 0.0), B.CCE_ERR_INVALID)):
        with pytest.raises(B.CCEError) as error:
            B.cce_orthogonalize_multi([x], coefficients=c)
        assert error.value.code == code
    with pytest.raises(B.CCEError):
        B.cce_orthogonalize_multi([x], eps=-1.0)
    with pytest.raises(B.CCEError):
        B.cce_orthogonalize_multi([x], workspace=torch.empty(255, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        B.cce_orthogonalize_multi([x], coefficients=(1.0, 2.0))
    p, m = torch.zeros_like(x), torch.zeros_like(x)
    handle = B.MuonTensors([x], [p], [m])
    for kw in (dict(lr=-1.0), dict(lr=1.0, momentum=1.0), dict(lr=math.nan)):
        with pytest.raises(B.CCEError):
            B.cce_muon_multi_step(handle, **kw)
    with pytest.raises(ValueError):
        B.MuonTensors([x], [p], [p])
    with pytest.raises(ValueError):
        B.MuonTensors([x], [p.view(6, 4)], [m])
    with pytest.raises(ValueError):
        handle.set_grads([x.view(6, 4)])
    with pytest.raises(ValueError):
        B.cce_grad_sumsq_multi(handle)
    with pytest.raises(ValueError):
        B.cce_adamw_multi_step(handle, 1, lr=0.1)
    with pytest.raises(ValueError):
        B.cce_muon_multi_step(B.OptimTensors([x.view(-1)]), lr=0.1)
    assert bool((p == 0).all()) and bool((m == 0).all())
