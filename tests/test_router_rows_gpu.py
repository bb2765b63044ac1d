"""What a row of the router gives is that row's alone, and what a call gives is tensors of their own."""
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


@pytest.mark.parametrize("N,E,k", [(4, 64, 4), (3000, 16, 2)])
def test_outputs_are_tensors_of_their_own(B, N, E, k):
    """Counts summed over ranks in place between a forward and a backward pass that saved the others; losses kept for a log."""
    x = torch.randn(N, E, device="cuda")

    class Route(torch.autograd.Function):
        @staticmethod
        def forward(ctx, logits):
            f = B.cce_router_forward(logits, k)
            ctx.save_for_backward(logits, f.indices, f.lse)
            ctx.counts = f.counts
            return f.weights, f.losses

        @staticmethod
        def backward(ctx, d_weights, d_losses):
            logits, indices, lse = ctx.saved_tensors
            return B.cce_router_backward(logits, indices, lse, ctx.counts, d_weights.contiguous(), d_losses.contiguous())

    f = B.cce_router_forward(x, k)
    assert len({t.untyped_storage().data_ptr() for t in f}) == 6 and f.losses.untyped_storage().nbytes() <= 64
    before = [t._version for t in f]
    f.counts.mul_(2)
    assert [t._version for t in f] == [v + (name == "counts") for name, v in zip(f._fields, before)]
    leaf = x.clone().requires_grad_()
    weights, losses = Route.apply(leaf)
    weights.grad_fn.counts.mul_(2)                                       # as after an all-reduce over two ranks of the same rows
    (weights.sum() + (losses * torch.tensor([0.1, 0.01], device="cuda")).sum()).backward()
    want = B.cce_router_backward(x, f.indices, f.lse, f.counts, torch.ones(N, k, device="cuda"), torch.tensor([0.1, 0.01], device="cuda"))
    assert torch.equal(leaf.grad, want)
