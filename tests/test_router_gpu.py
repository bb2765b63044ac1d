"""GPU parity of the router entry points with their oracle in 64 bits.

Tolerances (u = 2^-24, half a step of fp32).  exp of an argument d = logit - top (or - lse): the argument's rounding moves it by u |d|, the
factor log2 e by 2 u |d| more, exp2 itself and the rest by 4 u.  A row's sum of positive terms adds at most u for each of the 16 values of a
lane and the 6 steps between lanes.  So with d the row's largest finite |d| and e = (3 d + 32) u:
    weights      2 e + 4 u of themselves (numerator, sum, reciprocal and product)
    lse          e + 4 u |lse| (log of the sum, and the sum with top)
    prob_sums    2 e + 4 u + N / 8 u of themselves: sums of a lane's rows in fp32
    losses       balance as prob_sums, z 2 (e + 4 u |lse|) |lse|, and 4 u of the rounding at the end
    d_logits     p (2 (e + 4 u) + 24 u) times the sum of the magnitudes of what it is multiplied with, and bf16's 2^-8 of itself"""
import math

import numpy as np
import pytest
import torch

from oracle import router_oracle as R

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
IGN = -100
# N, E, k
SIZES = [(1, 1, 1), (1, 8, 2), (3, 2, 1), (5, 7, 7), (4, 64, 4), (33, 8, 2), (100, 16, 3), (65, 17, 5), (257, 60, 4), (130, 61, 6), (70, 128, 8), (33, 129, 9),
         (41, 256, 8), (19, 255, 32), (9, 300, 12), (7, 512, 8), (6, 513, 32), (5, 1023, 5), (5, 1024, 32), (6, 33, 32), (2100, 8, 1), (200, 96, 6), (150, 200, 8), (90, 264, 5), (400, 512, 7), (384, 20, 2), (385, 64, 3), (128, 200, 4), (129, 200, 4)]


@pytest.fixture(scope="module")
def B():
    from paper_2601_02609_amd import binding
    binding.lib()
    return binding


def _inputs(N, E, k, bf16, masked, seed=0, scale=2.0):
    rng = np.random.default_rng(seed + 7 * N + E + 31 * k)
    x = torch.from_numpy((rng.standard_normal((N, E)) * scale).astype(np.float32))
    if masked:
        x[torch.from_numpy(rng.random((N, E)) < masked)] = -math.inf
        if N > 3:
            x[N // 2] = -math.inf                                                 # a row without an expert
    x = x.bfloat16() if bf16 else x
    labels = torch.from_numpy(rng.integers(0, 1000, N).astype(np.int32))
    labels[torch.from_numpy(rng.random(N) < 0.2)] = IGN
    if N > 2:
        x[torch.nonzero(labels == IGN)[:1, 0]] = math.nan                         # padding may hold anything
    return x, labels


def _errors(x, f):
    """e of each row."""
    usable = np.isfinite(x) & f["p"].any(1)[:, None]
    top = np.max(np.where(usable, x, -np.inf), axis=1, keepdims=True)
    d = np.where(usable, np.where(usable, top, 0.0) - np.where(usable, x, 0.0), 0.0)
    return (3.0 * d.max(1) + 32.0) * U


def _check_forward(got, x, labels, k, renormalize=True):
    x = x.double().numpy()
    f = R.forward(x, k, None if labels is None else labels.numpy() != IGN, renormalize)
    e = _errors(x, f)
    np.testing.assert_array_equal(got.indices.cpu().numpy(), f["indices"])
    np.testing.assert_array_equal(got.counts.cpu().numpy(), f["counts"])
    w, lse, sums, losses = (t.cpu().numpy().astype(np.float64) for t in (got.weights, got.lse, got.prob_sums, got.losses))
    assert (np.abs(w - f["weights"]) <= (2 * e + 4 * U)[:, None] * f["weights"]).all()
    lse_off = e + 4 * U * np.abs(f["lse"])
    assert (np.abs(lse - f["lse"]) <= np.where(f["p"].any(1), lse_off, 0.0)).all()
    off = 2 * e.max() + 4 * U + len(x) / 8 * U
    assert (np.abs(sums - f["prob_sums"]) <= off * f["prob_sums"]).all()
    assert abs(losses[0] - f["losses"][0]) <= (off + 4 * U) * f["losses"][0]
    n = max(int(f["counts"][-1]), 1)
    assert abs(losses[1] - f["losses"][1]) <= (2 * lse_off * np.abs(f["lse"])).sum() / n + 4 * U * f["losses"][1]
    return f


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("masked", [0.0, 0.6])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_forward(B, size, masked, bf16):
    N, E, k = size
    x, labels = _inputs(N, E, k, bf16, masked)
    for renormalize in (True, False):
        got = B.cce_router_forward(x.cuda(), k, labels.cuda(), IGN, renormalize=renormalize)
        _check_forward(got, x, labels, k, renormalize)
    whole = torch.nan_to_num(x.float(), nan=0.0, neginf=-math.inf).to(x.dtype)
    _check_forward(B.cce_router_forward(whole.cuda(), k), whole, None, k)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("masked", [0.0, 0.6])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_backward(B, size, masked, bf16):
    N, E, k = size
    x, labels = _inputs(N, E, k, bf16, masked, seed=1)
    rng = np.random.default_rng(N + E)
    dw = rng.standard_normal((N, k)).astype(np.float32)
    dl = np.array([0.3, -0.02], dtype=np.float32)
    for renormalize, use_w, use_l in ((True, True, True), (False, True, True), (True, False, True), (True, True, False)):
        f = R.forward(x.double().numpy(), k, labels.numpy() != IGN, renormalize)
        e = _errors(x.double().numpy(), f)
        d_w = np.where(f["indices"] >= 0, dw, np.nan).astype(np.float32)           # never read where there is no expert
        got = B.cce_router_backward(x.cuda(), torch.from_numpy(f["indices"]).cuda(), torch.from_numpy(f["lse"].astype(np.float32)).cuda(),
                                    torch.from_numpy(f["counts"]).cuda(), torch.from_numpy(d_w).cuda() if use_w else None,
                                    torch.from_numpy(dl).cuda() if use_l else None, renormalize=renormalize)
        assert got.dtype == x.dtype
        dwu, dlu = (dw if use_w else 0 * dw), (dl if use_l else 0 * dl).astype(np.float64)
        xx = np.nan_to_num(x.double().numpy(), nan=0.0, neginf=-np.inf)
        want = R.backward(xx, f["indices"], f["counts"], dwu, dlu, renormalize)
        n = max(int(f["counts"][-1]), 1)
        chosen = f["indices"] >= 0
        at = np.maximum(f["indices"], 0)
        ps = np.where(chosen, np.take_along_axis(f["p"], at, 1), 0.0)
        s = np.where(f["p"].any(1), ps.sum(1), 1.0)[:, None] if renormalize else 1.0
        a = np.where(chosen, np.abs(dwu), 0.0)
        direct = np.zeros_like(xx)
        for q in range(k):
            np.add.at(direct, (np.arange(N), at[:, q]), np.where(chosen[:, q], ((a + (a * ps).sum(1, keepdims=True) / s) / s)[:, q], 0.0))
        beta = abs(dlu[0]) * E / (k * n * n) * f["counts"][:E]
        size_of = direct + beta + (a * ps).sum(1, keepdims=True) / s + (beta * f["p"]).sum(1, keepdims=True) + np.abs(2 * dlu[1] * f["lse"] / n)[:, None]
        off = f["p"] * ((4 * e + 32 * U)[:, None] * size_of) + (2.0 ** -8 if bf16 else 0.0) * np.abs(want) + (2.0 ** -133 if bf16 else 2.0 ** -149)
        d = np.abs(got.double().cpu().numpy() - want)
        assert (d <= off).all(), (renormalize, use_w, use_l, (d / off).max())


def test_ties_and_signed_zeros_go_to_the_lowest_index(B):
    for bf16 in (False, True):
        for E in (8, 64, 256, 1000):
            rng = np.random.default_rng(E)
            x = torch.from_numpy(rng.integers(-1, 2, (50, E)).astype(np.float32))
            x[::3] *= -1.0                                                        # -0 beside 0
            x = x.bfloat16() if bf16 else x
            k = min(E, 10)
            _check_forward(B.cce_router_forward(x.cuda(), k), x, None, k)


def test_values_that_differ_in_their_last_bits(B):
    """More alike than a sorting key with a column in it can tell, in some rows in their first places, in others at the border of the chosen ones."""
    for E, k in ((8, 2), (60, 4), (128, 8), (256, 7), (500, 8), (1000, 3)):
        rng = np.random.default_rng(E)
        near = 1.0 + np.stack([rng.permutation(E) for _ in range(40)]) * 2.0 ** -23
        far = rng.standard_normal((40, E))
        x = np.concatenate([near, -near, far, np.where(rng.random((40, E)) < k / E, 3.0 + far, near), np.where(rng.random((40, E)) < 0.5, far, -near)])
        x = torch.from_numpy(x[rng.permutation(len(x))].astype(np.float32))
        _check_forward(B.cce_router_forward(x.cuda(), k), x, None, k)


@pytest.mark.parametrize("E,k,bf16", [(60, 3, False), (256, 8, False), (64, 4, True), (256, 8, True), (512, 6, True)])
def test_values_that_are_no_numbers(B, E, k, bf16):
    x = torch.randn(40, E)
    x[3, 7] = math.nan
    x[4, 9], x[4, 2] = math.inf, math.nan
    x[5, 11] = -math.nan
    got = B.cce_router_forward(x.bfloat16().cuda() if bf16 else x.cuda(), k)
    idx = got.indices.cpu()
    assert idx[3, 0] == 7 and idx[4, 0] == 2 and idx[4, 1] == 9 and idx[5, 0] == 11
    bad = torch.zeros(40, dtype=torch.bool)
    bad[3:6] = True
    w = got.weights.cpu()
    assert bool(w[bad].isnan().all()) and bool(w[~bad].isfinite().all()) and bool(got.lse.cpu()[bad].isnan().all())
    assert bool(got.losses.isnan().all()) and int(got.counts[-1]) == 40 and int(got.counts[:-1].sum()) == 40 * k


@pytest.mark.parametrize("E,k", [(8, 2), (61, 6), (128, 6), (256, 8), (512, 8)])
def test_large_logits_and_many_rows(B, E, k):
    """Far more rows than the workgroups take at a time; logits whose exponentials fp32 does not hold."""
    N = 20011
    gen = torch.Generator(device="cuda").manual_seed(E)
    x = torch.randn(N, E, device="cuda", generator=gen) * 60.0
    labels = torch.randint(0, 9, (N,), device="cuda", generator=gen, dtype=torch.int32)
    got = B.cce_router_forward(x, k, labels, 4)
    live = labels != 4
    p = torch.softmax(x.double(), 1) * live[:, None]
    order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k].int()
    assert torch.equal(got.indices, torch.where(live[:, None], order, -1))
    counts = torch.bincount(order[live].flatten().long(), minlength=E)
    n = int(live.sum())
    assert torch.equal(got.counts[:E].long(), counts) and int(got.counts[E]) == n
    off = (6 * float((x.amax(1) - x.amin(1)).max()) + 68 + N / 8) * U
    assert bool(((got.prob_sums.double() - p.sum(0)).abs() <= off * p.sum(0)).all())
    lse = torch.logsumexp(x.double(), 1) * live
    assert bool(((got.lse.double() - lse).abs() <= (3 * 0 + 40 + 6 * lse.abs()) * U).all())
    want = E / (k * n * n) * float((counts * p.sum(0)).sum())
    assert abs(float(got.losses[0]) - want) <= (off + 4 * U) * want
    again = B.cce_router_forward(x, k, labels, 4)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


def test_nothing_beside_the_outputs_and_unaligned_memory(B):
    for bf16 in (False, True):
        for N, E, k in ((37, 64, 4), (50, 60, 3), (1300, 16, 2)):
            x, labels = _inputs(N, E, k, bf16, 0.3, seed=5)

            def odd(shape, dtype, fill):
                whole = torch.full((math.prod(shape) + 9,), fill, dtype=dtype, device="cuda")
                return whole, whole[1:1 + math.prod(shape)].view(*shape)

            xw, xd = odd((N, E), x.dtype, 0)
            xd.copy_(x)
            outs = [odd(s, d, 7) for s, d in (((N, k), torch.int32), ((N, k), torch.float32), ((N,), torch.float32), ((E + 1,), torch.int32),
                                              ((E,), torch.float32), ((2,), torch.float32))]
            ws = torch.full((int(B.lib().cce_router_workspace_bytes(N, E)) + 256,), 0xff, dtype=torch.uint8, device="cuda")
            out = B.RouterOutput(*(v for _, v in outs))
            got = B.cce_router_forward(xd, k, labels.cuda(), IGN, out=out, workspace=ws[:-256])
            _check_forward(got, x, labels, k)
            for w, v in outs:
                assert int(w[0]) == 7 and bool((w[1 + v.numel():] == 7).all())
            assert bool((ws[-256:] == 0xff).all())
            gw, gd = odd((N, E), x.dtype, 7)
            dw = torch.randn(N, k, device="cuda")
            dl = torch.tensor([0.1, 0.2], device="cuda")
            B.cce_router_backward(xd, got.indices, got.lse, got.counts, dw, dl, d_logits=gd)
            assert int(gw[0]) == 7 and bool((gw[1 + gd.numel():] == 7).all())
            same = B.cce_router_backward(x.cuda(), got.indices, got.lse, got.counts, dw, dl)
            assert torch.equal(same, gd)
            inplace = x.cuda()
            B.cce_router_backward(inplace, got.indices, got.lse, got.counts, dw, dl, d_logits=inplace)
            assert torch.equal(same, inplace)


def test_gradient_is_that_of_differences(B):
    """Through both entry points: the derivative along a random direction."""
    N, E, k = 64, 40, 4
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(N, E, device="cuda", generator=gen)
    dw = torch.randn(N, k, device="cuda", generator=gen)
    dl = torch.tensor([0.5, 0.05], device="cuda")
    f = B.cce_router_forward(x, k)
    g = B.cce_router_backward(x, f.indices, f.lse, f.counts, dw, dl)
    v = torch.randn(N, E, device="cuda", generator=gen)

    def value(y):
        return R.total(y.double().cpu().numpy(), f.indices.cpu().numpy(), f.counts.cpu().numpy(), dw.cpu().numpy(), dl.cpu().numpy(), True)

    h = 1e-5
    want = (value(x.double() + h * v.double()) - value(x.double() - h * v.double())) / (2 * h)
    # central differences in 64 bits: h^2 times third derivatives; the gradient's own error is some 100 u of the sum of magnitudes
    assert abs(float((g.double() * v.double()).sum()) - want) <= 200 * U * float((g.double() * v.double()).abs().sum()) + 1e-6


def test_counts_of_other_ranks(B):
    """Two halves of a batch, their counts summed, give the gradient of the whole."""
    N, E, k = 96, 32, 2
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(N, E, device="cuda", generator=gen)
    dl = torch.tensor([1.0, 0.1], device="cuda")
    whole = B.cce_router_forward(x, k)
    want = B.cce_router_backward(x, whole.indices, whole.lse, whole.counts, None, dl)
    halves = [B.cce_router_forward(h.contiguous(), k) for h in x.chunk(2)]
    counts = halves[0].counts + halves[1].counts
    assert torch.equal(counts, whole.counts)
    for i, h in enumerate(x.chunk(2)):
        got = B.cce_router_backward(h.contiguous(), halves[i].indices, halves[i].lse, counts, None, dl)
        assert torch.equal(got, want.chunk(2)[i])
    n = float(counts[-1])
    sums = halves[0].prob_sums + halves[1].prob_sums
    assert abs(float(E / (k * n * n) * (counts[:-1].double() * sums.double()).sum()) - float(whole.losses[0])) <= 1e-5 * float(whole.losses[0])


def test_captured_and_replayed(B):
    N, E, k = 3000, 64, 4
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(N, E, device="cuda", generator=gen)
    dw, dl = torch.randn(N, k, device="cuda", generator=gen), torch.tensor([0.5, 0.05], device="cuda")
    ws = torch.empty(int(B.lib().cce_router_workspace_bytes(N, E)), dtype=torch.uint8, device="cuda")
    out = B.cce_router_forward(x, k, workspace=ws)
    d = B.cce_router_backward(x, out.indices, out.lse, out.counts, dw, dl)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.cce_router_forward(x, k, out=out, workspace=ws)
        B.cce_router_backward(x, out.indices, out.lse, out.counts, dw, dl, d_logits=d)
    for i in range(3):
        x.copy_(torch.randn(N, E, device="cuda", generator=gen))
        want = B.cce_router_forward(x, k)
        want_d = B.cce_router_backward(x, want.indices, want.lse, want.counts, dw, dl)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)) and torch.equal(d, want_d), i
        ws.fill_(0xff)


def test_indexes_out_of_range_are_passed_over(B):
    x = torch.randn(5, 12, device="cuda")
    f = B.cce_router_forward(x, 3)
    bad = f.indices.clone()
    bad[2, 1], bad[3, 2], bad[4, 0] = 12, 2 ** 31 - 1, -5
    g = B.cce_router_backward(x, bad, f.lse, f.counts, torch.ones(5, 3, device="cuda"), None)
    fine = bad.clone()
    fine[2, 1] = fine[3, 2] = -1
    assert torch.equal(g, B.cce_router_backward(x, fine, f.lse, f.counts, torch.ones(5, 3, device="cuda"), None)) and bool((g[4] == 0).all())


def test_refusals(B):
    x = torch.randn(5, 12, device="cuda")
    for k, code in ((0, B.CCE_ERR_INVALID), (13, B.CCE_ERR_INVALID)):
        with pytest.raises(B.CCEError) as error:
            B.cce_router_forward(x, k)
        assert error.value.code == code
    with pytest.raises(B.CCEError) as error:
        B.cce_router_forward(torch.randn(2, 64, device="cuda"), 33)
    assert error.value.code == B.CCE_ERR_UNSUPPORTED
    with pytest.raises(B.CCEError) as error:
        B.cce_router_forward(torch.randn(2, 1025, device="cuda"), 2)
    assert error.value.code == B.CCE_ERR_UNSUPPORTED
    for bad in (x.half(), x.t(), x.cpu(), x[0]):
        with pytest.raises((ValueError, TypeError)):
            B.cce_router_forward(bad, 2)
    with pytest.raises(ValueError):
        B.cce_router_forward(x, 2, torch.zeros(4, dtype=torch.int32, device="cuda"))
    with pytest.raises(B.CCEError):
        B.cce_router_forward(x, 2, workspace=torch.empty(4, dtype=torch.uint8, device="cuda"))
    f = B.cce_router_forward(x, 2)
    with pytest.raises(ValueError):
        B.cce_router_backward(x, f.indices, f.lse, f.counts[:-1], None, None)
    with pytest.raises(ValueError):
        B.cce_router_backward(x, f.indices, f.lse, f.counts, torch.zeros(5, 3, device="cuda"), None)
