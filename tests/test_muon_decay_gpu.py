"""Decay of a Muon step.  The entry decays by its matrix's own rate, 1 - lr lr_scale weight_decay; the optimizer as it is published, and as torch
has it, by 1 - lr weight_decay whatever the matrix's shape: that is weight_decay / lr_scale here, as the header and the list say."""
import math

import numpy as np
import pytest
import torch

from oracle import muon_oracle as M

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
ABC = (3.4445, -4.7750, 2.0315)
SHAPES = [(16, 180), (64, 64), (300, 40), (200, 700), (1400, 560)]
LR, WD, MU = 0.02, 0.1, 0.95


@pytest.fixture(scope="module")
def B():
    from paper_2601_02609_amd import binding
    binding.lib()
    return binding


def _state(seed):
    rng = np.random.default_rng(seed)
    return [[torch.from_numpy((rng.standard_normal(s) * scale).astype(np.float32)).cuda() for s in SHAPES] for scale in (0.02, 1e-3, 5e-4)]


def _published(B, grads, params, momentum):
    scale = [0.2 * math.sqrt(max(s)) for s in SHAPES]
    return B.MuonTensors(grads, params, momentum, lr_scale=scale, weight_decay=[WD / x for x in scale])


def test_decay_alone_is_torchs(B):
    """Gradients of zeros: the update is zero and decay is all that a step does.  Off by the rounding of weight_decay / lr_scale, of the two
    products and of 1 - their product, and of the product with the parameter, in torch's step and in this one: 2 * (3 lr wd + 2) 2^-24."""
    p, g, m = _state(0)
    leaves = [torch.nn.Parameter(x.clone()) for x in p]
    for x in leaves:
        x.grad = torch.zeros_like(x)
    optimizer = torch.optim.Muon(leaves, lr=LR, weight_decay=WD, momentum=MU, nesterov=True, adjust_lr_fn="match_rms_adamw")
    start = [x.clone() for x in p]
    handle = _published(B, [torch.zeros_like(x) for x in p], p, [torch.zeros_like(x) for x in p])
    optimizer.step()
    B.cce_muon_multi_step(handle, lr=LR, momentum=MU)
    for x, y, z in zip(p, leaves, start):
        assert bool(((x - y).abs() <= 2 * (3 * LR * WD + 2) * U * z.abs()).all())
        assert bool((x != z).any())


def test_step_is_the_published_rule(B):
    """Nesterov momentum, the orthogonalised direction in 64 bits, its learning rate with the shape's factor, decay without it.  What the header
    says of a result: 2^-9 of its 2-norm; the parameter's own roundings, 4 * 2^-24 of |param| + |update|."""
    p, g, m = _state(1)
    start, grads, before = ([x.cpu().numpy().astype(np.float64) for x in xs] for xs in (p, g, m))
    B.cce_muon_multi_step(_published(B, g, p, m), lr=LR, momentum=MU)
    for got, p0, g0, m0, shape in zip(p, start, grads, before, SHAPES):
        buffer = MU * m0 + (1 - MU) * g0
        update = LR * 0.2 * math.sqrt(max(shape)) * M.orthogonalize(MU * buffer + (1 - MU) * g0, ABC, 5, 1e-7)
        off = np.linalg.norm(got.cpu().numpy() - ((1 - LR * WD) * p0 - update))
        assert off <= 2.0 ** -9 * np.linalg.norm(update) + 4 * U * (np.linalg.norm(p0) + np.linalg.norm(update))
