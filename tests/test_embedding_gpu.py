"""GPU parity of the embedding lookup and its gradient with the fp64 oracle.

Tolerances, from the arithmetic: the lookup is one fp32 product rounded to bf16, the same bits as NumPy's.  A sum of
n fp32 terms in any order is off by at most (n - 1) 2^-24 of the sum of their magnitudes; the scale and the
addition to dW round once more each: (n + 2) 2^-24 of what the oracle calls the size."""
import numpy as np
import pytest
import torch

from oracle import embedding_oracle as E
from paper_2601_02609_amd import inputs as I
from tests.gpu_util import bf16_dev

pytestmark = pytest.mark.gpu
IGN = -100


@pytest.fixture(scope="module")
def B():
    from paper_2601_02609_amd import binding
    binding.lib()
    return binding


def _bits(x):
    return I.f32_to_bf16_bits(np.asarray(x, dtype=np.float32))


def _tokens(rng, N, V, kind, ignore):
    if kind == "zipf":
        p = np.arange(1, V + 1) ** -1.2
        t = rng.choice(V, N, p=p / p.sum())
    elif kind == "one":
        t = np.full(N, V - 1)
    elif kind == "runs":                                                    # every token 31 times: sums that end inside any piece
        t = rng.permutation(np.arange(N) // 31 % V)
    else:
        t = rng.integers(0, V, N)
    t = t.astype(np.int32)
    t[rng.random(N) < ignore] = IGN
    return t


def _guarded(shape, dtype):
    """A tensor in the middle of a larger one, and a check that its surroundings are as they were."""
    n = int(np.prod(shape))
    whole = torch.full((n + 2048,), 7.0, dtype=dtype, device="cuda")
    return whole[1024:1024 + n].view(shape), lambda: bool((whole[:1024] == 7).all() and (whole[1024 + n:] == 7).all())


@pytest.mark.parametrize("N,D,V,kind,ignore,scale", [
    (1, 8, 1, "uniform", 0.0, 1.0), (1, 896, 5000, "uniform", 0.0, 29.933), (3, 24, 7, "zipf", 0.4, -0.5), (257, 64, 1000, "uniform", 0.1, 1.0),
    (1000, 896, 3001, "zipf", 0.15, 29.933), (63, 4096, 100, "zipf", 0.3, 64.0), (5, 65536, 3, "uniform", 0.0, 2.0), (2049, 1032, 33, "one", 0.2, 1.0),
    (100, 72, 50, "uniform", 1.0, 3.0)])
def test_lookup_is_the_rounded_product(B, N, D, V, kind, ignore, scale):
    rng = np.random.default_rng(N + D)
    w, t = _bits(rng.standard_normal((V, D))), _tokens(rng, N, V, kind, ignore)
    print(f"[lookup] N={N} D={D} V={V}", flush=True)
    out, intact = _guarded((N, D), torch.bfloat16)
    B.cce_embedding_forward(torch.from_numpy(t).cuda(), bf16_dev(w), IGN, scale=scale, out=out)
    got = out.view(torch.int16).cpu().numpy().view(np.uint16)
    want = np.zeros((N, D), dtype=np.uint16)
    ok = E.takes_part(t, V, IGN)
    want[ok] = _bits(np.float32(scale) * I.bf16_bits_to_f32(w[t[ok]]))
    assert np.array_equal(got, want) and intact()
    assert np.array_equal(E.forward(I.bf16_bits_to_f32(w[:, :8]).astype(np.float64), t, IGN, 1.0)[ok], I.bf16_bits_to_f32(w[t[ok], :8]))


def _gradient_case(B, N, D, V, kind, ignore, scale, accumulate, seed=0):
    rng = np.random.default_rng(N + D + V + seed)
    t = _tokens(rng, N, V, kind, ignore)
    dy = _bits(rng.standard_normal((N, D)) * np.exp(rng.uniform(-3, 3, (N, 1))))
    ok = E.takes_part(t, V, IGN)
    dy[~ok] = 0x7FC0                                                        # NaN where no token takes part
    dw0 = rng.standard_normal((V, D)).astype(np.float32)
    dw, intact = _guarded((V, D), torch.float32)
    dw.copy_(torch.from_numpy(dw0) if accumulate else torch.full((V, D), float("nan")))
    print(f"[gradient] N={N} D={D} V={V} {kind} accumulate={accumulate}", flush=True)
    need = B.embedding_workspace_bytes(N, D, V)
    ws = torch.full((need + 4096,), 171, dtype=torch.uint8, device="cuda")
    B.cce_embedding_backward(torch.from_numpy(t).cuda(), bf16_dev(dy), V, IGN, scale=scale, d_weight=dw, accumulate_dw=accumulate,
                             workspace=ws[:need])
    assert bool((ws[need:] == 171).all())
    got = dw.cpu().numpy()
    want, size = E.backward(I.bf16_bits_to_f32(dy).astype(np.float64), t, V, IGN, float(np.float32(scale)), dw0 if accumulate else None)
    count = np.bincount(t[ok], minlength=V)
    assert np.all(np.abs(got - want) <= (count[:, None] + 2) * 2.0 ** -24 * size)
    assert intact()
    assert np.array_equal(got[count == 0], (dw0 if accumulate else np.zeros_like(dw0))[count == 0])


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("N,D,V,kind,ignore,scale", [
    (1, 8, 1, "uniform", 0.0, 1.0), (2, 8, 300, "one", 0.0, 1.0), (257, 64, 1000, "uniform", 0.1, 1.0), (63, 16, 5, "zipf", 0.3, 0.5),
    (64, 72, 7, "uniform", 0.0, 1.0), (1000, 24, 9, "zipf", 0.1, -1.5), (5000, 896, 3001, "zipf", 0.15, 29.933), (2048, 128, 151936, "zipf", 0.0, 1.0),
    (4097, 1032, 1, "one", 0.05, 1.0), (3000, 512, 40, "zipf", 0.0, 1.0), (300, 8192, 50, "zipf", 0.2, 1.0), (7, 65536, 3, "uniform", 0.0, 1.0),
    (1500, 256, 4000, "runs", 0.0, 1.0), (10000, 520, 257, "uniform", 0.5, 1.0), (100, 64, 50, "uniform", 1.0, 1.0), (2500, 1024, 300, "runs", 0.4, 1.0),
    (40000, 40, 20000, "zipf", 0.1, 1.0), (33000, 8, 2, "uniform", 0.0, 1.0), (1025, 3584, 600000 // 512, "zipf", 0.0, 1.0)])
def test_gradient_matches_oracle(B, N, D, V, kind, ignore, scale, accumulate):
    _gradient_case(B, N, D, V, kind, ignore, scale, accumulate)


@pytest.mark.parametrize("V", [255, 256, 257, 511, 512, 262143, 262144, 262145, 600001])
def test_gradient_at_vocabulary_borders(B, V):
    _gradient_case(B, 700, 16, V, "uniform", 0.1, 1.0, True)
    _gradient_case(B, 700, 16, V, "one", 0.1, 1.0, False)


@pytest.mark.parametrize("N,D,V,hot", [(1_100_003, 8, 70000, 0.5), (300_001, 64, 700, 0.0), (70_000, 264, 200_000, 0.9), (1_048_577, 16, 1, 0.0)])
def test_gradient_of_many_tokens(B, N, D, V, hot):
    """Ranges of a wavefront beyond 16 bits, and more of a slice's tokens in one than it notes: whole numbers, whose sums
    fp32 holds."""
    rng = np.random.default_rng(N)
    t = rng.integers(0, V, N).astype(np.int32)
    t[rng.random(N) < hot] = min(5, V - 1)
    t[rng.random(N) < 0.05] = IGN
    dy = rng.integers(-4, 5, (N, D))
    ok = E.takes_part(t, V, IGN)
    want = np.stack([np.bincount(t[ok], weights=dy[ok, j], minlength=V) for j in range(D)], axis=1)
    assert np.abs(dy).sum(0).max() < 2 ** 24
    print(f"[gradient] N={N} D={D} V={V}", flush=True)
    td, dyd = torch.from_numpy(t).cuda(), torch.from_numpy(dy).cuda().bfloat16()
    for accumulate in (False, True):
        dw, intact = _guarded((V, D), torch.float32)
        dw.fill_(3.0)
        B.cce_embedding_backward(td, dyd, V, IGN, scale=2.0, d_weight=dw, accumulate_dw=accumulate)
        assert np.array_equal(dw.cpu().numpy(), 2.0 * want + (3.0 if accumulate else 0.0)) and intact()


def test_tokens_outside_the_matrix_are_reported(B):
    V, D = 30, 64
    t = np.array([0, 30, 29, -1, IGN, 5, 2 ** 31 - 1, -2 ** 31], dtype=np.int32)
    rng = np.random.default_rng(5)
    w, dy = _bits(rng.standard_normal((V, D))), _bits(rng.standard_normal((len(t), D)))
    status = torch.full((1,), 64, dtype=torch.int32, device="cuda")
    td = torch.from_numpy(t).cuda()
    out = B.cce_embedding_forward(td, bf16_dev(w), IGN, status=status)
    assert int(status) == 64 | B.CCE_STATUS_BAD_TOKEN                       # OR-ed in, nothing cleared
    ok = E.takes_part(t, V, IGN)
    assert ok.tolist() == [True, False, True, False, False, True, False, False]
    assert torch.equal(out.cpu()[torch.from_numpy(~ok)], torch.zeros((~ok).sum(), D, dtype=torch.bfloat16))
    status.zero_()
    dw = B.cce_embedding_backward(td, bf16_dev(dy), V, IGN, status=status)
    assert int(status) == B.CCE_STATUS_BAD_TOKEN
    want, _ = E.backward(I.bf16_bits_to_f32(dy).astype(np.float64), t, V, IGN)
    assert np.array_equal(dw.cpu().numpy(), want)                           # single rows: no rounding
    status.zero_()
    good = torch.from_numpy(np.array([IGN, 3, 29], dtype=np.int32)).cuda()
    B.cce_embedding_forward(good, bf16_dev(w), IGN, status=status)
    B.cce_embedding_backward(good, bf16_dev(dy[:3]), V, IGN, status=status)
    assert int(status) == 0
    B.cce_embedding_forward(td, bf16_dev(w), IGN)                           # no status word: nothing to report to
    # an ignore_index inside the vocabulary takes its token out
    out = B.cce_embedding_forward(good, bf16_dev(w), 29, status=status)
    assert int(status) == B.CCE_STATUS_BAD_TOKEN and not bool(out[2].any()) and bool(out[1].any())


@pytest.mark.parametrize("N", [1, 64, 700, 1025, 5000, 40001])
@pytest.mark.parametrize("bad", [-1, 100, -2 ** 31, 2 ** 31 - 1])
def test_one_bad_token_anywhere_is_reported(B, N, bad):
    """In one launch and in three, at either end: by both calls, and not without one."""
    V, D = 100, 64
    dy = torch.ones(N, D, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(V, D, dtype=torch.bfloat16, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for at in (None, 0, N // 2, N - 1):
        t = torch.full((N,), IGN, dtype=torch.int32, device="cuda")
        t[N // 3] = 7
        if at is not None:
            t[at] = bad
        for call in (lambda: B.cce_embedding_forward(t, w, IGN, status=status), lambda: B.cce_embedding_backward(t, dy, V, IGN, status=status)):
            status.zero_()
            call()
            assert int(status) == (0 if at is None else B.CCE_STATUS_BAD_TOKEN), at


def test_gradient_is_the_same_in_every_run_and_with_any_workspace(B):
    rng = np.random.default_rng(6)
    N, D, V = 6000, 256, 500
    t = torch.from_numpy(_tokens(rng, N, V, "zipf", 0.1)).cuda()
    dy = torch.randn(N, D, device="cuda").bfloat16()
    a = B.cce_embedding_backward(t, dy, V, IGN)
    need = B.embedding_workspace_bytes(N, D, V)
    for fill, extra in ((0, 0), (255, 0), (127, 4096)):
        ws = torch.full((need + extra,), fill, dtype=torch.uint8, device="cuda")
        assert torch.equal(a, B.cce_embedding_backward(t, dy, V, IGN, workspace=ws))
    # a larger batch's workspace serves a smaller one
    big = torch.full((B.embedding_workspace_bytes(20000, D, V),), 255, dtype=torch.uint8, device="cuda")
    assert torch.equal(a, B.cce_embedding_backward(t, dy, V, IGN, workspace=big))


def test_gradient_of_the_lookup_against_differences(B):
    """<dy, y(W + h P) - y(W - h P)> / 2h = <dW, P>: the lookup is linear, so differences of exact bf16 values are exact
    up to the fp32 sums (2^-24 of each term, N D terms)."""
    rng = np.random.default_rng(7)
    N, D, V = 300, 64, 40
    t = torch.from_numpy(_tokens(rng, N, V, "zipf", 0.1)).cuda()
    w = torch.randint(-8, 9, (V, D), device="cuda").bfloat16()
    p = torch.randint(-8, 9, (V, D), device="cuda").bfloat16()
    dy = torch.randint(-8, 9, (N, D), device="cuda").bfloat16()
    up, down = (B.cce_embedding_forward(t, w + s * p, IGN, scale=2.0).double() for s in (1, -1))
    dw = B.cce_embedding_backward(t, dy, V, IGN, scale=2.0).double()
    assert float(((up - down) / 2 * dy.double()).sum()) == float((dw * p.double()).sum())


def test_rows_beyond_32_bit_offsets(B):
    """2.2 G values of dW and of W: the last rows' offsets pass 2^31 values and 2^32 bytes."""
    D, V = 8192, 270000
    w = torch.zeros(V, D, dtype=torch.bfloat16, device="cuda")
    w[V - 1] = torch.randn(D, device="cuda").bfloat16()
    t = torch.tensor([V - 1, 0, V - 1, V - 2], dtype=torch.int32, device="cuda")
    out = B.cce_embedding_forward(t, w)
    assert torch.equal(out[0], w[V - 1]) and torch.equal(out[2], w[V - 1]) and not bool(out[1].any())
    del w
    dw = torch.full((V, D), 3.0, device="cuda")
    B.cce_embedding_backward(t, out, V, d_weight=dw)
    assert torch.equal(dw[V - 1], 2 * out[0].float()) and not bool(dw[:V - 1].any())


def test_binding_refuses(B):
    t = torch.zeros(4, dtype=torch.int32, device="cuda")
    w = torch.zeros(10, 64, dtype=torch.bfloat16, device="cuda")
    dy = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    for bad in (t.long(), t[::2], t.view(2, 2)):
        with pytest.raises(ValueError):
            B.cce_embedding_forward(bad, w)
    for bad in (w.float(), w[:, ::2], w.t()):
        with pytest.raises(ValueError):
            B.cce_embedding_forward(t, bad)
    with pytest.raises(ValueError):
        B.cce_embedding_forward(t, w, out=torch.empty(4, 64, device="cuda"))
    with pytest.raises(ValueError):
        B.cce_embedding_backward(t, dy, 10, accumulate_dw=True)
    with pytest.raises(ValueError):
        B.cce_embedding_backward(t, dy, 10, d_weight=torch.empty(9, 64, device="cuda"))
    with pytest.raises(ValueError):
        B.cce_embedding_backward(t, dy, 10, status=torch.zeros(1, device="cuda"))
    with pytest.raises(B.CCEError):
        B.cce_embedding_backward(t, dy, 10, workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))
    with pytest.raises(B.CCEError):                                         # rows of 12 values are not 16-byte chunks
        B.cce_embedding_forward(t, torch.zeros(10, 12, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(B.CCEError):
        B.cce_embedding_backward(t[:0], dy[:0], 10)


# ------------------------------------------------------------------ sizes from which other variants run
def _whole_tokens(N, V, hot, seed, rows=None):
    """Tokens of `rows` (all of them, if not given), both ends of the matrix among them; one of them has a share `hot` of the positions."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows = torch.arange(V, device="cuda", dtype=torch.int32) if rows is None else rows
    t = rows[torch.randint(0, len(rows), (N,), device="cuda", generator=gen)]
    t[torch.rand(N, device="cuda", generator=gen) < hot] = rows[len(rows) // 2]
    t[torch.rand(N, device="cuda", generator=gen) < 0.1] = IGN
    for i, at in enumerate((0, N // 2, N - 1)[:N]):
        t[at] = (0, V - 1, 0)[i]
    return t


def _exact_gradient(B, N, D, V, accumulate, t, seed=0):
    """Whole numbers, whose sums fp32 holds: the bits of the sum in 64 bits.  NaN in rows that take no part."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dy = torch.randint(-4, 5, (N, D), device="cuda", generator=gen).bfloat16()
    ok = t != IGN
    assert int(torch.bincount(t[ok].long()).max()) * 4 < 2 ** 22
    want = torch.zeros(V, D, dtype=torch.float64, device="cuda").index_add_(0, t[ok].long(), dy[ok].double())
    want = (2.0 * want + (3.0 if accumulate else 0.0)).float()
    dy[~ok] = float("nan")
    dw, intact = _guarded((V, D), torch.float32)
    dw.fill_(3.0 if accumulate else float("nan"))
    print(f"[gradient] N={N} D={D} V={V} accumulate={accumulate}", flush=True)
    need = B.embedding_workspace_bytes(N, D, V)
    ws = torch.full((need + 4096,), 171, dtype=torch.uint8, device="cuda")
    B.cce_embedding_backward(t, dy, V, IGN, scale=2.0, d_weight=dw, accumulate_dw=accumulate, workspace=ws[:need])
    assert torch.equal(dw, want) and intact() and bool((ws[need:] == 171).all())


@pytest.mark.parametrize("N,D,V", [(12287, 8192, 500), (12288, 8192, 500), (97601, 1032, 3000), (12_582_917, 8, 70)])
def test_lookup_of_outputs_that_the_caches_do_not_hold(B, N, D, V):
    """192 MiB of y and more, and one row less: the rounded products, bit for bit."""
    assert (N * D * 2 >= 192 << 20) == (N != 12287)
    t = _whole_tokens(N, V, 0.2, N)
    w = (torch.randn(V, D, device="cuda") * 0.3).bfloat16()
    out, intact = _guarded((N, D), torch.bfloat16)
    print(f"[lookup] N={N} D={D} V={V}", flush=True)
    B.cce_embedding_forward(t, w, IGN, scale=-1.7, out=out)
    want = (w.float() * float(np.float32(-1.7))).bfloat16()[t.clamp(min=0).long()]
    want[t == IGN] = 0
    assert torch.equal(out.view(torch.int16), want.view(torch.int16)) and intact()


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("N,D,V", [(16400, 4104, 40), (16352, 4104, 40), (3000, 4104, 16400), (17000, 4096, 17000), (600_001, 120, 560_000)])
def test_gradient_of_what_the_caches_do_not_hold(B, N, D, V, accumulate):
    """128 MiB of dy (and a little less), 256 MiB of dW, both; a third of the rows get zeros."""
    t = _whole_tokens(N, V, 0.3, N + D, torch.arange(V, device="cuda", dtype=torch.int32)[torch.arange(V, device="cuda") % 3 != 1])
    _exact_gradient(B, N, D, V, accumulate, t)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("V", [1, 255, 256, 257, 163839, 163840, 163841, 327680, 327681])
def test_gradient_at_the_borders_of_the_slices(B, V, accumulate):
    """640 rows of the matrix are a slice's most: in one launch and in three, both ends of the matrix named."""
    for N in (700, 2100, 9000):
        _exact_gradient(B, N, 16, V, accumulate, _whole_tokens(N, V, 0.2, N + V))


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("N,D", [(1024, 64), (1025, 64), (1024, 1024), (682, 1032), (683, 1032), (1024, 2048), (1024, 2056), (16, 65536), (33, 65536)])
def test_gradient_where_one_launch_ends(B, N, D, accumulate):
    for hot in (0.0, 1.0):
        _exact_gradient(B, N, D, 300, accumulate, _whole_tokens(N, 300, hot, N + D))


@pytest.mark.parametrize("accumulate", [False, True])
def test_three_launches_beyond_32_bit_offsets_of_dw(B, accumulate):
    """2.2 G values of dW with 3000 tokens: what is written, and that nothing else is."""
    N, D, V = 3000, 8192, 270000
    rows = torch.cat([torch.arange(600), torch.arange(V - 600, V), torch.arange(262100, 262200)]).cuda().int()
    t = _whole_tokens(N, V, 0.1, 9, rows)
    dy = torch.randint(-4, 5, (N, D), device="cuda").bfloat16()
    ok, fill = t != IGN, 3.0 if accumulate else 0.0
    named, at = torch.unique(t[ok].long(), return_inverse=True)
    want = torch.zeros(len(named), D, dtype=torch.float64, device="cuda").index_add_(0, at, dy[ok].double()).float() + fill
    dw = torch.full((V, D), 3.0, device="cuda")
    B.cce_embedding_backward(t, dy, V, IGN, d_weight=dw, accumulate_dw=accumulate)
    assert torch.equal(dw[named], want)
    dw[named] = fill
    assert bool((dw == fill).all())


def test_rows_beyond_32_bit_offsets_of_y(B):
    """2.2 G values of y and of dy: the lookup's rows, and their gradient, which is a row's count times itself."""
    N, D, V = 270000, 8192, 50
    t = _whole_tokens(N, V, 0.3, 10)
    w = torch.randint(-3, 4, (V, D), device="cuda").bfloat16()
    y = B.cce_embedding_forward(t, w, IGN)
    for first in range(0, N, 30000):
        part = slice(first, first + 30000)
        want = w[t[part].clamp(min=0).long()]
        want[t[part] == IGN] = 0
        assert torch.equal(y[part], want), first
    dw = B.cce_embedding_backward(t, y, V, IGN)
    assert torch.equal(dw, torch.bincount(t[t != IGN].long(), minlength=V)[:, None] * w.float())
