"""What a row of the router gives is that row's alone."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2601_02609_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("E,k", [(8, 2), (16, 4), (64, 4), (60, 7), (128, 8), (256, 8), (500, 6), (1000, 8), (64, 9)])
def test_a_rows_bits_do_not_depend_on_its_neighbours(B, E, k, bf16):
    """Ties at the border of the chosen ones, values that are no numbers, masked and ignored rows between rows of plain numbers: these stay as
    they are beside others of their kind."""
    N = 96
    gen = torch.Generator().manual_seed(E)
    x = torch.randn(N, E, generator=gen)
    others = torch.randint(-1, 2, (N, E), generator=gen).float()
    others[1::8, 3] = math.nan
    others[3::8, 2] = math.inf
    others[5::8] = -math.inf
    mixed = x.clone()
    mixed[1::2] = others[1::2]
    labels = torch.zeros(N, dtype=torch.int32)
    labels[7::8] = -100
    if bf16:
        x, mixed = x.bfloat16(), mixed.bfloat16()
    for renormalize in (True, False):
        alone = B.cce_router_forward(x.cuda(), k, renormalize=renormalize)
        beside = B.cce_router_forward(mixed.cuda(), k, labels.cuda(), renormalize=renormalize)
        for name in ("indices", "weights", "lse"):
            a, b = getattr(alone, name)[::2], getattr(beside, name)[::2]
            assert torch.equal(a.view(torch.int32), b.view(torch.int32)), name
