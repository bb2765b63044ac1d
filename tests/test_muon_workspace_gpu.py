"""The workspace of the matrices' calls: exactly as many bytes as asked for, whatever they hold before, and nothing behind them touched; lists
whose launches take every kind of tile and part."""
import pytest
import torch

pytestmark = pytest.mark.gpu
ABC = (3.4445, -4.7750, 2.0315)
EPS = 1e-7
GUARD = 1 << 16
LISTS = {
    "one workgroup each": [(5, 7), (30, 40), (64, 100), (100, 128)],
    "thin": [(16, 3000), (40, 5000), (2100, 33), (64, 16500)],
    "tiles": [(130, 140), (300, 200), (257, 450), (65, 449)],
    "two steps as one": [(512, 1280), (1400, 500), (513, 2000)],
    "split sums of few rows": [(100, 4096), (6000, 300)],
    "last tiles split": [(1090, 1100)] * 5 + [(2048, 2048)],
    "all": [(5, 7), (64, 100), (40, 5000), (300, 200), (512, 1280), (100, 4096), (1090, 1100), (0, 3)],
}


@pytest.fixture(scope="module")
def B():
    from paper_2601_02609_amd import binding
    binding.lib()
    return binding


def _matrices(shapes):
    gen = torch.Generator(device="cuda").manual_seed(len(shapes))
    return [torch.randn(s, device="cuda", generator=gen) for s in shapes]


def _check(got, g):
    """bf16 results within the header's 2^-9 of the 2-norm, and bf16's 2^-8 of each value."""
    x = g.double() / (torch.linalg.norm(g.double()) + EPS)
    x = x if len(x) <= x.shape[1] else x.T.contiguous()
    for a, b, c in [ABC] * 5:
        gram = x @ x.T
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    x = x if g.shape[0] <= g.shape[1] else x.T.contiguous()
    assert float(torch.linalg.norm(got.double() - x)) <= (2.0 ** -9 + 2.0 ** -8) * float(torch.linalg.norm(x)), g.shape


def _results(B, matrices, need, fill):
    ws = torch.full((need + GUARD,), fill, dtype=torch.uint8, device="cuda")
    ws[need:] = 0xa5
    out = B.cce_orthogonalize_multi(matrices, workspace=ws[:need])
    assert bool((ws[need:] == 0xa5).all())
    return out


@pytest.mark.parametrize("name", LISTS)
def test_asked_for_bytes_are_enough_and_may_hold_anything(B, name):
    x = _matrices(LISTS[name])
    params, momentum = [torch.zeros_like(t) for t in x], [torch.zeros_like(t) for t in x]
    handle = B.MuonTensors(x, params, momentum)
    need = B.muon_workspace_bytes(handle)
    first, second = (_results(B, x, need, fill) for fill in (0xff, 0x00))             # NaN in every type, and zeros
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    with pytest.raises(B.CCEError):
        B.cce_orthogonalize_multi(x, workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
    ws = torch.full((need + GUARD,), 0xff, dtype=torch.uint8, device="cuda")
    B.cce_muon_multi_step(handle, lr=1.0, momentum=0.0, nesterov=False, workspace=ws[:need])
    assert bool((ws[need:] == 0xff).all())
    for o, p, g in zip(first, params, x):
        if g.numel():
            _check(o, g)
            assert torch.equal(o, (-p).bfloat16())


def test_split_tiles_of_a_few_rows(B):
    """Matrices of 65 to 128 rows beside some of 4096: their tiles are among the split ones of a product of r x r, a slice a part."""
    shapes = [(4096, 4096)] * 2 + [(100, 1000), (65, 500), (128, 470), (500, 70)]
    x = _matrices(shapes)
    out = B.cce_orthogonalize_multi(x)
    for o, g in zip(out, x):
        _check(o, g)
    again = B.cce_orthogonalize_multi(x)
    assert all(torch.equal(a, b) for a, b in zip(out, again))


@pytest.mark.parametrize("shape,count", [((1900, 5000), 5), ((5700, 2048), 5), ((600, 1600), 3), ((1100, 3000), 2)], ids=lambda x: "x".join(map(str, x)) if isinstance(x, tuple) else str(x))
def test_whole_products_of_two_steps_taken_as_one(B, shape, count):
    """The last product of the two steps, which is not mirrored: tiles of 256 x 256 with the last ones in parts of their sums, ragged ones among them, and
    tiles of 128 x 128.  Each matrix of its own values, and the same bits again."""
    x = _matrices([shape] * count)
    x = [t * (1.0 + i) for i, t in enumerate(x)]
    out = B.cce_orthogonalize_multi(x)
    for o, g in zip(out, x):
        _check(o, g)
    assert all(torch.equal(a, b) for a, b in zip(out, B.cce_orthogonalize_multi(x)))
